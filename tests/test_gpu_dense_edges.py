"""GPU tests of the dense operators where errors hide: the last digits of gelu, the one rounding of dz, every tile of the products, layer
norms wider than the row kernels, sums over as many tokens as there may be.

U: half a step of fp32, relative to the value; HALF: half a step of the output's type."""
import numpy as np
import pytest
import torch
from scipy import special

import paper_2602_16249_amd as aff
from oracle import dense
from product_sizes import SIZES
from test_gpu_dense import Guarded, _close, _norm_bwd_bounds, _norm_inputs, _shifted, _stored

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


# ------------------------------------------------------------------------------------------------------------------ gelu

def _gelu_points(dtype):
    z = torch.cat([torch.linspace(-12, 12, 48001), torch.linspace(-0.01, 0.01, 2001)]).to(TYPES[dtype])
    return z.cuda().view(-1, 1), z.double().numpy()


# Relative errors in units of U.  The exponent z^2 / 2: z z and its product with -1/2 log2(e) are rounded once each, 2 U (z^2 / 2) = z^2 U of
# the result together; the hardware's exponential is off by 2 U (one step); the polynomial's fit by 0.7 (fp32) or 4 (bf16); t = 1 / (1 + c |z|) by
# the hardware's reciprocal, 2 U, which counts 2.1 (fp32) or 2.7 times (bf16), 4.2 or 5.4; the last of the sum's roundings, sum of |terms| / value
# 3.6 at t = 1, count 7; s t, its product with e, 1 - tail and z cdf one each.  In all z^2 + 18 in fp32, z^2 + 22.4 in bf16: z^2 + 24 is taken.
ROUNDINGS = 24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gelu_to_the_last_digits(dtype):
    """Far into the negative tail, where gelu is small: relative to its own size."""
    t, z = _gelu_points(dtype)
    got, _ = aff.affmae_linear_fwd(t, torch.ones(1, 1, dtype=t.dtype, device="cuda"), act="gelu")
    ref = z * special.ndtr(z)
    tol = (z * z + ROUNDINGS) * U * np.abs(ref)
    off = np.abs(got.double().cpu().numpy()[:, 0] - ref)
    over = off > tol + HALF[dtype] * (np.abs(ref) + tol)
    assert not over.any(), (int(over.sum()), z[over][0], off[over][0] / abs(ref[over][0]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slope_of_gelu_to_the_last_digits(dtype):
    """The slope is cdf + z density, two terms of either sign: relative to the sum of their sizes."""
    t, z = _gelu_points(dtype)
    one = torch.ones(1, 1, dtype=t.dtype, device="cuda")
    got = aff.affmae_linear_bwd(None, one, torch.ones_like(t), t, act="gelu", want_dweight=False)["dx"]
    cdf, part = special.ndtr(z), z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    ref = cdf + part
    tol = (z * z + ROUNDINGS) * U * (cdf + np.abs(part))
    half = HALF[dtype] if dtype == "f32" else 2 * HALF[dtype] + HALF[dtype] ** 2  # (bf16: dz and the gradient, one rounding each)
    off = np.abs(got.double().cpu().numpy()[:, 0] - ref)
    over = off > tol + half * (np.abs(ref) + tol)
    assert not over.any(), (int(over.sum()), z[over][0], off[over][0])


@pytest.mark.parametrize("G", [1, 4])
def test_gelu_behind_a_norm(G):
    """The norm's own activation: constant channels of +-1 make xhat +-1 (eps 1e-12), gamma carries the value."""
    z = np.linspace(-9, 9, 64).astype(np.float32)
    x = torch.ones(40, 1, 64, device="cuda")
    x[..., 1::2] = -1
    sign = x[0, 0].cpu().numpy()
    gamma = torch.from_numpy(z * sign).cuda()
    out, mean, rstd = aff.affmae_norm_fwd(x, gamma, torch.zeros(64, device="cuda"), G, 1e-12, act="gelu")
    zd = z.astype(np.float64)
    ref = zd * special.ndtr(zd)
    # xhat is off by 4 U, z then by as much: z |slope| / |gelu| <= 1 + z^2 for z < 0
    tol = ((1 + zd * zd) * 5 + zd * zd + ROUNDINGS) * U * np.abs(ref)
    assert bool((mean == 0).all()) and (np.abs(out.double().cpu().numpy()[:, 0] - ref) <= tol + U * np.abs(ref)).all()


def test_gelu_of_infinities():
    z = torch.tensor([[float("inf")], [float("nan")], [3e38], [-3e38], [0.0]], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    got, _ = aff.affmae_linear_fwd(z, one, act="gelu")
    assert got[0, 0] == float("inf") and bool(torch.isnan(got[1, 0])) and got[2, 0] == z[2, 0] and got[3, 0] == 0 and got[4, 0] == 0
    g = aff.affmae_linear_bwd(None, one, torch.ones_like(z), z, act="gelu", want_dweight=False)["dx"]
    assert bool(torch.isnan(g[1, 0])) and g[2, 0] == 1 and g[3, 0] == 0 and g[4, 0] == 0.5


# ---------------------------------------------------------------------------------------------- one rounding of dz, no other

@pytest.mark.parametrize("rows,cin,cout", [(1030, 136, 264), (700, 65, 191), (16400, 776, 2312)])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_bf16_gradients_are_the_products_of_dz_rounded_once(rows, cin, cout, p):
    """dx and dweight against products in 64 bits of dz rounded to bf16, dbias against the sum of dz as it is.  dz (in front of the mask's
    factor, which the sums are multiplied by) is off by (z^2 + 24) U of the sum of the slope's two terms; where that spans a border of the
    rounding, by the step between the two."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    normal = lambda *shape, std=1.0: (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()
    x, w, dout, pre = normal(rows, cin), normal(cout, cin, std=cin ** -0.5), normal(rows, cout), normal(rows, cout, std=1.1)
    rng = torch.tensor([77, 5], dtype=torch.int64, device="cuda")
    got = aff.affmae_linear_bwd(x, w, dout, pre, act="gelu", p=p, rng=rng)
    z, d = pre.double(), dout.double()
    if p:
        d = torch.where(torch.from_numpy(dense.keep((rows, cout), p, 77, 5)).cuda(), d, 0.0)
    f = 1.0 / (1.0 - float(np.float32(p)))
    cdf, part = 0.5 * torch.special.erfc(-z * 2 ** -0.5), z * torch.exp(-0.5 * z * z) * (2 * np.pi) ** -0.5
    dz = d * (cdf + part)
    e = (z * z + 25) * U * d.abs() * (cdf + part.abs())
    lo, hi = (dz - e).float().bfloat16().double(), (dz + e).float().bfloat16().double()
    r, step = dz.float().bfloat16().double(), (hi - lo).abs()
    assert float((step > 0).double().mean()) < 0.01  # (so that nearly every value's rounding is known)
    a = r.abs() + step
    wd, xd = w.double(), x.double()
    rt, st, at = r.t().contiguous(), step.t().contiguous(), a.t().contiguous()
    for k, ref, tol in (("dx", f * (r @ wd), f * (step @ wd.abs() + 2 * U * (cout + 6) * (a @ wd.abs()))),
                        ("dweight", f * (rt @ xd), f * (st @ xd.abs() + 2 * U * (rows + 6) * (at @ xd.abs()))),
                        ("dbias", f * dz.sum(0), f * (e.sum(0) + 2 * U * (rows + 6) * dz.abs().sum(0)))):
        over = (got[k].double() - ref).abs() > tol + HALF["bf16"] * (ref.abs() + tol)
        assert not bool(over.any()), f"{k}: {int(over.sum())} of {over.numel()} off"


# ------------------------------------------------------------ norms whose channels' sums are taken over runs of images, backward

WIDE = [  # dtype, B, N, C, groups: pieces of 16 bytes down to single values, shares of a group, whole groups beside each other
    ("bf16", 2100, 1, 8200, 1), ("bf16", 2100, 1, 8196, 1), ("bf16", 1030, 1, 8198, 1), ("bf16", 1030, 1, 8201, 1), ("f32", 2100, 1, 4100, 1),
    ("f32", 1030, 1, 4098, 1), ("f32", 4100, 1, 4097, 1), ("bf16", 300, 1, 20000, 1), ("bf16", 2300, 3, 2600, 1), ("bf16", 2100, 3, 302, 2),
    ("f32", 6200, 2, 302, 2), ("bf16", 2049, 2, 4112, 2), ("bf16", 8200, 33, 65, 1),
]


@pytest.mark.parametrize("dtype,B,N,C,G", WIDE)
def test_norm_backward_over_runs_of_images(dtype, B, N, C, G):
    name = ["silu", "none", "relu"][(B + N + C) % 3]
    d = _norm_inputs(dtype, B, N, C, seed=11)
    v = {k: a[1] for k, a in d.items()}
    _, mean, rstd = dense.norm_fwd(v["x"], v["gamma"], v["beta"], G, 1e-5)
    (tm, mean), (tr, rstd) = _stored(mean, "f32"), _stored(rstd, "f32")
    ref, bounds = _norm_bwd_bounds(v, mean, rstd, G, name, True, dtype)
    g = {"dx": Guarded((B, N, C), TYPES[dtype]), "dgamma": Guarded((C,), torch.float32), "dbeta": Guarded((C,), torch.float32)}
    args = (d["x"][0], d["gamma"][0], d["beta"][0], tm, tr, d["dout"][0], G)
    need = aff.load_library().affmae_norm_bwd_workspace_bytes(B, N, C, G, 1 if dtype == "bf16" else 0)
    space = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
    aff.affmae_norm_bwd(*args, act=name, grads={k: o.t for k, o in g.items()}, workspace=space[256:256 + need])
    for k in g:
        _close(g[k].t, ref[k], bounds[k], k)
        g[k].check()
    assert bool((space[:256] == 77).all()) and bool((space[256 + need:] == 77).all())
    again = aff.affmae_norm_bwd(*args, act=name)
    assert all(torch.equal(again[k], g[k].t) for k in g)
    bare = aff.affmae_norm_bwd(args[0], None, None, *args[3:])  # (no gamma: no sums of channels)
    assert set(bare) == {"dx"} and bool(torch.isfinite(bare["dx"]).all())


# ------------------------------------------------------------------------------------------------ every tile of the products

@pytest.mark.parametrize("dtype,rows,cin,cout,made,shift", SIZES)
def test_every_tile_of_the_products(dtype, rows, cin, cout, made, shift):
    """Forward and gradients against products in 64 bits on the device, value by value, in outputs with guards around them.  gelu is off by
    (z^2 + 24) U of |z| Phi(-|z|) and 3 U |z| of what is left, its slope by as much of Phi(-|z|) + |z| phi(z) and 2 U; a sum of n terms by 2 U (n + 5)
    of their sizes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + cin)
    normal = lambda *shape, std=1.0: _shifted((torch.randn(*shape, generator=g, device="cuda") * std).to(TYPES[dtype]), shift)
    x, w, b, r, dout, pre = (normal(rows, cin), normal(cout, cin, std=cin ** -0.5), normal(cout, std=0.3), normal(rows, cout), normal(rows, cout),
                             normal(rows, cout, std=1.5))
    act, p = ("gelu", 0.2) if made else ("none", 0.0)
    rng = torch.tensor([2602, 41], dtype=torch.int64, device="cuda")
    f = 1.0 / (1.0 - float(np.float32(p)))
    keep = torch.from_numpy(dense.keep((rows, cout), p, 2602, 41)).cuda() if made else None
    half = HALF[dtype]

    def close(got, ref, tol, what):
        got.check()
        over = ~((got.t.double() - ref).abs() <= tol + half * (ref.abs() + tol))
        assert not bool(over.any()), f"{what}: {int(over.sum())} of {over.numel()} off, first at {over.nonzero()[0].tolist()}"

    tail = lambda z: 0.5 * torch.special.erfc(z.abs() * 2 ** -0.5)
    cdf = lambda z: 0.5 * torch.special.erfc(-z * 2 ** -0.5)
    density = lambda z: torch.exp(-0.5 * z * z) * (2 * np.pi) ** -0.5
    guarded = lambda *shape: Guarded(shape, TYPES[dtype], shift)

    out, zo = guarded(rows, cout), guarded(rows, cout)
    aff.affmae_linear_fwd(x, w, b, r, act=act, p=p, rng=rng, out=out.t, pre=zo.t)
    xd, wt = x.double(), w.double().t().contiguous()
    z = xd @ wt + b.double()
    e = 2 * U * (cin + 5) * (xd.abs() @ wt.abs() + b.double().abs())
    close(zo, z, e, "pre")
    if made:
        branch = torch.where(keep, z * cdf(z) * f, 0.0)
        e = f * (1.13 * e + U * ((z * z + 24) * z.abs() * tail(z) + 3 * z.abs())) + 4 * U * f * z.abs()
    else:
        branch = z
    ref = r.double() + branch
    close(out, ref, e + U * (r.double().abs() + ref.abs()), "out")
    del out, zo, xd, wt, z, e, branch, ref

    dx, dw, db = guarded(rows, cin), guarded(cout, cin), guarded(cout)
    aff.affmae_linear_bwd(x, w, dout, pre if made else None, act=act, p=p, rng=rng, grads={"dx": dx.t, "dweight": dw.t, "dbias": db.t})
    d, z = dout.double(), pre.double()
    if made:
        d = torch.where(keep, d * f, 0.0)
        e = U * d.abs() * ((z * z + 24) * (tail(z) + z.abs() * density(z)) + 2) + 4 * U * d.abs()
        dz = d * (cdf(z) + z * density(z))
        e0, e = e, e + (half * (dz.abs() + e) if dtype == "bf16" else 0.0)  # dz rounded once as an operand, not for dbias
    else:
        dz, e = d, torch.zeros_like(d)
        e0 = e
    a = dz.abs() + e
    wd, xd = w.double(), x.double()
    close(dx, dz @ wd, e @ wd.abs() + 2 * U * (cout + 6) * (a @ wd.abs()), "dx")
    zt, et, at = dz.t().contiguous(), e.t().contiguous(), a.t().contiguous()
    close(dw, zt @ xd, et @ xd.abs() + 2 * U * (rows + 6) * (at @ xd.abs()), "dweight")
    close(db, dz.sum(0), e0.sum(0) + 2 * U * (rows + 6) * (dz.abs() + e0).sum(0), "dbias")


# -------------------------------------------------------------------------------- sums over as many tokens as there may be

@pytest.mark.parametrize("B,N,C,G,serial", [
    # terms that a sum adds one after another: by a thread, over the threads of a column, over a run of parts and over the runs.  What a launch does:
    (1, 2 ** 31 - 2 ** 16, 1, 1, 2 ** 13 + 256 + 64 + 16),  # 1024 workgroups of 2097088 tokens, 256 threads a column; 16 runs of 64 parts
    (2, 9_000_005, 128, 4, 1099 + 16 + 64 + 16),            # 2 x 512 workgroups of 17579 tokens, 16 threads a column; the same
    (16_777_215, 1, 136, 1, 2048 + 8 + 32 + 32),            # 1024 workgroups, 8 rows at a time; 32 runs of 32 parts
])
def test_channel_sums_of_very_many_tokens(B, N, C, G, serial):
    """-1, 1, -1, ... and dout = x: the terms of dgamma are all rstd, so that it is tokens x rstd up to `serial` roundings (a part of the
    thousand that went missing would be 1e-3 of it); dbeta's are whole numbers, exact up to 2^24 and then off by one an addition."""
    x = torch.ones(B, N, C, dtype=torch.bfloat16, device="cuda")
    flat = x.view(-1)
    flat[::2] = -1
    gamma, beta = torch.full((C,), 3.0, device="cuda").bfloat16(), torch.zeros(C, device="cuda").bfloat16()
    out, mean, rstd = aff.affmae_norm_fwd(x, gamma, beta, G, eps=1e-5)
    assert bool((mean == 0).all()) and bool((rstd == rstd.view(-1)[0]).all())
    got = aff.affmae_norm_bwd(x, gamma, beta, mean, rstd, x, G, grads={"dx": out})
    tokens = B * N
    r = float(rstd.view(-1)[0])
    assert float((got["dgamma"].double() / (tokens * r) - 1).abs().max()) <= (serial + 8) * U
    # (an odd number of channels: a channel's signs alternate from token to token; an even one: they are the same in all)
    want = torch.zeros(C) if C % 2 else torch.where(torch.arange(C) % 2 == 0, -tokens, tokens)
    assert float((got["dbeta"].double().cpu() - want.double()).abs().max()) <= (0 if tokens % 2 == 0 and C % 2 else 4)
