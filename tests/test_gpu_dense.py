"""GPU parity of the dense operators (matrix product with epilogue, group norm with activation, dropout) against the plain 64-bit
implementations on the same stored values, value by value.

Bounds: U is half a step of fp32 and half(dtype) half a step of the output's type, relative to the value.  A sum of n terms in
fp32 is off by at most 2 U (n + 4) times the sum of the terms' absolute values, whatever the order (2 U instead of U: matrix
instructions may truncate).  The activations are off by at most 8 U times (1 + |z|) (device exponential and reciprocal, polynomial
of the normal distribution)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2602_16249_amd as aff
from oracle import dense

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
SLOPE = 1.13  # the largest slope of the activations
SEED = (2602, 41)


def _stored(a, dtype):
    """A device tensor of the storage type, and the values that it holds."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPES[dtype])
    return t.cuda(), t.double().numpy()


class Guarded:
    """An output inside a larger buffer whose other elements have to stay as they were; `shift` elements off its alignment."""

    def __init__(self, shape, dtype, shift=0):
        self.n = int(np.prod(shape))
        self.buf = torch.full((self.n + 256,), 77.0, dtype=dtype, device="cuda")
        self.lo = 128 + shift
        self.t = self.buf[self.lo:self.lo + self.n].view(shape)

    def check(self):
        assert bool((self.buf[:self.lo] == 77).all()) and bool((self.buf[self.lo + self.n:] == 77).all()), "written outside"


def _shifted(t, shift):
    """The same values `shift` elements off the allocation's alignment."""
    if not shift or t is None:
        return t
    buf = torch.empty(t.numel() + shift, dtype=t.dtype, device=t.device)
    v = buf[shift:].view(t.shape)
    v.copy_(t)
    return v


def _close(got, ref, tol, what):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, what
    over = ~(np.abs(got - ref) <= tol)
    if over.any():
        i = tuple(int(v) for v in np.argwhere(over)[0])
        raise AssertionError(f"{what}: {int(over.sum())} of {over.size} off, first at {i}: {got[i]} for {ref[i]}, bound {np.broadcast_to(tol, ref.shape)[i]}")


def _rng(call=SEED[1]):
    return torch.tensor([SEED[0], call], dtype=torch.int64, device="cuda")


# ------------------------------------------------------------------------------------------------------------- products

def _linear_inputs(dtype, rows, cin, cout, seed=0):
    g = np.random.default_rng(seed + rows * 7919 + cin * 31 + cout)
    a = {"x": g.normal(size=(rows, cin)), "w": g.normal(size=(cout, cin)) / np.sqrt(cin), "b": g.normal(size=cout) * 0.3,
         "r": g.normal(size=(rows, cout)), "dout": g.normal(size=(rows, cout)), "pre": g.normal(size=(rows, cout)) * 1.5}
    return {k: _stored(v, dtype) for k, v in a.items()}


def _linear_fwd_bounds(v, name, p, use_bias, use_res, dtype):
    cin = v["x"].shape[1]
    b, r = (v["b"] if use_bias else None), (v["r"] if use_res else None)
    out, z = dense.linear_fwd(v["x"], v["w"], b, r, name, p, SEED)
    f = 1.0 / (1.0 - float(np.float32(p)))
    dz = 2 * U * (cin + 5) * (np.abs(v["x"]) @ np.abs(v["w"]).T + (np.abs(b) if use_bias else 0))
    branch = f * (SLOPE * dz + (0 if name == "none" else 8 * U * (1 + np.abs(z)))) + 4 * U * f * np.abs(z)
    d = branch + (U * (np.abs(r) + np.abs(out)) if use_res else 0)
    return out, z, d + HALF[dtype] * (np.abs(out) + d), dz + HALF[dtype] * (np.abs(z) + dz)


LINEAR = [  # rows, cin, cout
    (1, 1, 1), (1, 64, 192), (2, 3, 5), (16, 8, 8), (17, 64, 64), (63, 72, 40), (64, 2304, 768), (65, 128, 130), (129, 100, 301), (128, 33, 64),
    (257, 256, 256), (300, 768, 63), (1000, 64, 1), (1025, 192, 64), (2049, 24, 200), (4100, 96, 260), (515, 520, 516), (700, 7, 9),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", LINEAR)
def test_linear_forward(dtype, rows, cin, cout):
    d = _linear_inputs(dtype, rows, cin, cout)
    v = {k: a[1] for k, a in d.items()}
    name = ["none", "relu", "gelu", "silu"][(rows + cin + cout) % 4]
    p = [0.0, 0.25][(rows + cout) % 2]
    use_bias, use_res = (rows + cin) % 3 != 0, (cin + cout) % 3 != 0
    out, z, tol, ztol = _linear_fwd_bounds(v, name, p, use_bias, use_res, dtype)
    go, gp = Guarded((rows, cout), TYPES[dtype]), Guarded((rows, cout), TYPES[dtype])
    got, pre = aff.affmae_linear_fwd(d["x"][0], d["w"][0], d["b"][0] if use_bias else None, d["r"][0] if use_res else None, act=name, p=p, rng=_rng(),
                                     out=go.t, pre=gp.t)
    _close(got, out, tol, "out")
    _close(pre, z, ztol, "pre")
    go.check()
    gp.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("p", [0.0, 0.7])
@pytest.mark.parametrize("rows,cin,cout", [(130, 64, 192), (20, 96, 72), (300, 36, 45)])
def test_linear_forward_epilogues(dtype, name, p, rows, cin, cout):
    d = _linear_inputs(dtype, rows, cin, cout, 1)
    out, _, tol, _ = _linear_fwd_bounds({k: a[1] for k, a in d.items()}, name, p, True, True, dtype)
    got, pre = aff.affmae_linear_fwd(d["x"][0], d["w"][0], d["b"][0], d["r"][0], act=name, p=p, rng=_rng() if p else None)
    assert pre is None
    _close(got, out, tol, "out")
    # onto the residual stream in place
    onto = d["r"][0].clone()
    again, _ = aff.affmae_linear_fwd(d["x"][0], d["w"][0], d["b"][0], onto, act=name, p=p, rng=_rng() if p else None, out=onto)
    assert again is onto and torch.equal(onto, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_linear_of_tensors_off_their_alignment(dtype, shift):
    rows, cin, cout = 200, 64, 96
    d = _linear_inputs(dtype, rows, cin, cout, 2)
    v = {k: a[1] for k, a in d.items()}
    s = {k: _shifted(a[0], shift) for k, a in d.items()}
    out, z, tol, ztol = _linear_fwd_bounds(v, "gelu", 0.25, True, True, dtype)
    go, gp = Guarded((rows, cout), TYPES[dtype], shift), Guarded((rows, cout), TYPES[dtype], shift)
    aff.affmae_linear_fwd(s["x"], s["w"], s["b"], s["r"], act="gelu", p=0.25, rng=_rng(), out=go.t, pre=gp.t)
    _close(go.t, out, tol, "out")
    _close(gp.t, z, ztol, "pre")
    ref, bounds = _linear_bwd_bounds(v, "gelu", 0.25, dtype)
    g = {"dx": Guarded((rows, cin), TYPES[dtype], shift), "dweight": Guarded((cout, cin), TYPES[dtype], shift), "dbias": Guarded((cout,), TYPES[dtype], shift)}
    aff.affmae_linear_bwd(s["x"], s["w"], s["dout"], s["pre"], act="gelu", p=0.25, rng=_rng(), grads={k: o.t for k, o in g.items()})
    for o in (go, gp, *g.values()):
        o.check()
    for k in g:
        _close(g[k].t, ref[k], bounds[k], k)


def _linear_bwd_bounds(v, name, p, dtype):
    f = 1.0 / (1.0 - float(np.float32(p)))
    dz = dense.linear_dz(v["dout"], v["pre"], name, p, SEED)
    ref = {"dx": dz @ v["w"], "dweight": dz.T @ v["x"], "dbias": dz.sum(0)}
    e = 4 * U * np.abs(dz)
    if name != "none":
        e = e + 8 * U * f * np.abs(v["dout"]) * (1 + np.abs(v["pre"]))
    if dtype == "bf16" and (name != "none" or p):
        e = e + HALF["bf16"] * (np.abs(dz) + e)
    rows, cout = dz.shape
    a = np.abs(dz) + e
    d = {"dx": e @ np.abs(v["w"]) + 2 * U * (cout + 5) * (a @ np.abs(v["w"])),
         "dweight": e.T @ np.abs(v["x"]) + 2 * U * (rows + 5) * (a.T @ np.abs(v["x"])),
         "dbias": e.sum(0) + 2 * U * (rows + 5) * a.sum(0)}
    return ref, {k: t + HALF[dtype] * (np.abs(ref[k]) + t) for k, t in d.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", LINEAR)
def test_linear_backward(dtype, rows, cin, cout):
    d = _linear_inputs(dtype, rows, cin, cout, 3)
    v = {k: a[1] for k, a in d.items()}
    name = ["gelu", "none", "silu", "relu", "none"][(rows + cin + cout) % 5]
    p = [0.0, 0.25][(rows + cin) % 2]
    ref, bounds = _linear_bwd_bounds(v, name, p, dtype)
    g = {"dx": Guarded((rows, cin), TYPES[dtype]), "dweight": Guarded((cout, cin), TYPES[dtype]), "dbias": Guarded((cout,), TYPES[dtype])}
    args = (d["x"][0], d["w"][0], d["dout"][0], d["pre"][0] if name != "none" else None)
    aff.affmae_linear_bwd(*args, act=name, p=p, rng=_rng(), grads={k: o.t for k, o in g.items()})
    for k in g:
        _close(g[k].t, ref[k], bounds[k], k)
        g[k].check()
    # each gradient alone, and the same bits again
    both = aff.affmae_linear_bwd(*args, act=name, p=p, rng=_rng(), want_dbias=False)
    assert set(both) == {"dx", "dweight"}
    one = aff.affmae_linear_bwd(None, args[1], args[2], args[3], act=name, p=p, rng=_rng(), want_dweight=False)
    other = aff.affmae_linear_bwd(args[0], None, args[2], args[3], act=name, p=p, rng=_rng(), want_dx=False)
    assert set(one) == {"dx"} and set(other) == {"dweight", "dbias"}
    for k, t in (("dx", both["dx"]), ("dx", one["dx"]), ("dweight", both["dweight"]), ("dweight", other["dweight"]), ("dbias", other["dbias"])):
        assert torch.equal(t, g[k].t), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("p", [0.0, 0.6])
def test_linear_backward_slopes(dtype, name, p):
    d = _linear_inputs(dtype, 333, 40, 88, 4)
    d["pre"][0][:2] = 0  # where relu has its corner
    d["pre"][1][:2] = 0
    ref, bounds = _linear_bwd_bounds({k: a[1] for k, a in d.items()}, name, p, dtype)
    got = aff.affmae_linear_bwd(d["x"][0], d["w"][0], d["dout"][0], d["pre"][0], act=name, p=p, rng=_rng() if p else None)
    for k in got:
        _close(got[k], ref[k], bounds[k], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_of_many_rows(dtype):
    """Sums over more rows than one workgroup adds up."""
    rows, cin, cout = 40001, 64, 72
    d = _linear_inputs(dtype, rows, cin, cout, 5)
    v = {k: a[1] for k, a in d.items()}
    ref, bounds = _linear_bwd_bounds(v, "gelu", 0.0, dtype)
    got = aff.affmae_linear_bwd(d["x"][0], d["w"][0], d["dout"][0], d["pre"][0], act="gelu")
    for k in got:
        _close(got[k], ref[k], bounds[k], k)
    again = aff.affmae_linear_bwd(d["x"][0], d["w"][0], d["dout"][0], d["pre"][0], act="gelu")
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("rows,cin,cout", [(16400, 776, 2312), (65552, 264, 264), (8200, 392, 1160), (20008, 264, 136), (8201, 767, 1023), (9000, 520, 1157), (16400, 2300, 1000)])
def test_linear_of_large_tiles(rows, cin, cout):
    """Sizes at which the larger tiles are taken, a little beyond whole tiles and slices, against products in 64 bits on the device."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    normal = lambda *shape, std=1.0: (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()
    x, w, b, r, dout, pre = (normal(rows, cin), normal(cout, cin, std=cin ** -0.5), normal(cout, std=0.3), normal(rows, cout), normal(rows, cout),
                             normal(rows, cout, std=1.5))
    p, f = 0.2, 1.0 / (1.0 - float(np.float32(0.2)))
    keep = torch.from_numpy(dense.keep((rows, cout), p, *SEED)).cuda()
    cdf = lambda z: 0.5 * torch.special.erfc(-z * 2 ** -0.5)
    half = HALF["bf16"]

    def close(got, ref, tol, what):
        over = ~((got.double() - ref).abs() <= tol + half * (ref.abs() + tol))
        assert not bool(over.any()), f"{what}: {int(over.sum())} of {over.numel()} off, first at {over.nonzero()[0].tolist()}"

    out, z = aff.affmae_linear_fwd(x, w, b, r, act="gelu", p=p, rng=_rng(), want_pre=True)
    xd, wt = x.double(), w.double().t().contiguous()
    rz = xd @ wt + b.double()
    dz = 2 * U * (cin + 5) * (xd.abs() @ wt.abs() + b.double().abs())
    close(z, rz, dz, "pre")
    branch = torch.where(keep, rz * cdf(rz) * f, 0.0)
    d = f * (SLOPE * dz + 8 * U * (1 + rz.abs())) + 4 * U * f * rz.abs() + U * (r.double().abs() + (r.double() + branch).abs())
    close(out, r.double() + branch, d, "out")
    del xd, wt, rz, dz, branch, d
    got = aff.affmae_linear_bwd(x, w, dout, pre, act="gelu", p=p, rng=_rng())
    pd = pre.double()
    z = torch.where(keep, dout.double() * f, 0.0) * (cdf(pd) + pd * torch.exp(-0.5 * pd * pd) * (2 * np.pi) ** -0.5)
    e = 4 * U * z.abs() + 8 * U * f * dout.double().abs() * (1 + pd.abs())
    e = e + half * (z.abs() + e)
    a = z.abs() + e
    wd, xd = w.double(), x.double()
    close(got["dx"], z @ wd, e @ wd.abs() + 2 * U * (cout + 5) * (a @ wd.abs()), "dx")
    zt, et, at = z.t().contiguous(), e.t().contiguous(), a.t().contiguous()
    close(got["dweight"], zt @ xd, et @ xd.abs() + 2 * U * (rows + 5) * (at @ xd.abs()), "dweight")
    close(got["dbias"], zt.sum(1), et.sum(1) + 2 * U * (rows + 5) * at.sum(1), "dbias")


@pytest.mark.parametrize("rows,cin,cout", [(3001, 1281, 1283), (3000, 1024, 1537), (2500, 1281, 1152), (20001, 65, 191)])
def test_linear_backward_of_odd_rows(rows, cin, cout):
    """bf16 rows of an odd length, of which large calls write copies: nothing but the gradients and the workspace is written."""
    d = _linear_inputs("bf16", rows, cin, cout, 7)
    ref, bounds = _linear_bwd_bounds({k: a[1] for k, a in d.items()}, "none", 0.0, "bf16")
    g = {"dx": Guarded((rows, cin), torch.bfloat16), "dweight": Guarded((cout, cin), torch.bfloat16), "dbias": Guarded((cout,), torch.bfloat16)}
    need = aff.load_library().affmae_linear_bwd_workspace_bytes(rows, cin, cout, 0, 0.0, 1, 1, 1)
    space = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")  # 256 bytes around it
    x, w, dout = (d[k][0] for k in ("x", "w", "dout"))
    before = [t.clone() for t in (x, w, dout)]
    aff.affmae_linear_bwd(x, w, dout, grads={k: o.t for k, o in g.items()}, workspace=space[256:256 + need])
    for k in g:
        _close(g[k].t, ref[k], bounds[k], k)
        g[k].check()
    assert bool((space[:256] == 77).all()) and bool((space[256 + need:] == 77).all())
    assert all(torch.equal(a, b) for a, b in zip(before, (x, w, dout)))
    one = aff.affmae_linear_bwd(None, w, dout, want_dweight=False)
    other = aff.affmae_linear_bwd(x, None, dout, want_dx=False)
    assert all(torch.equal(t, g[k].t) for k, t in (*one.items(), *other.items()))


def test_linear_leading_dimensions_and_values_that_are_not_finite():
    d = _linear_inputs("f32", 24, 16, 20, 6)
    x, w, b = (d[k][0] for k in "xwb")
    flat, _ = aff.affmae_linear_fwd(x, w, b)
    got, pre = aff.affmae_linear_fwd(x.view(2, 3, 4, 16), w, b, want_pre=True)
    assert got.shape == (2, 3, 4, 20) and torch.equal(got.view(24, 20), flat) and torch.equal(pre, got)
    one, _ = aff.affmae_linear_fwd(x[0], w, b)
    assert one.shape == (20,) and torch.equal(one, flat[0])
    # a row with an infinity and one with a NaN: these rows' values, no others
    bad = x.clone()
    bad[3, 5], bad[9, 0] = float("inf"), float("nan")
    got, _ = aff.affmae_linear_fwd(bad, w, b)
    ref = bad.double() @ w.double().t()
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isinf(got), torch.isinf(ref))
    clean = [i for i in range(24) if i not in (3, 9)]
    assert torch.equal(got[clean], flat[clean])
    # dropped values are replaced whatever they are
    keep = torch.from_numpy(dense.keep((24, 20), 0.5, *SEED)).cuda()
    got, _ = aff.affmae_linear_fwd(bad, w, b, p=0.5, rng=_rng())
    assert bool((got[~keep] == 0).all())


# ------------------------------------------------------------------------------------------------------------ group norm

NORM = [  # B, N, C, groups
    (1, 1, 1, 1), (3, 1, 8, 1), (5, 1, 64, 1), (130, 1, 256, 1), (7, 1, 100, 1), (33, 1, 768, 1), (9, 1, 2304, 1), (2, 1, 5000, 1), (4, 1, 96, 4),
    (2, 1, 20000, 1), (2, 17, 24, 3), (3, 50, 33, 11), (2, 1000, 64, 8), (1, 4097, 96, 12), (2, 300, 40, 1), (1, 70, 2056, 1), (65, 2, 16, 16),
    (3, 700, 12, 12), (1, 9, 4112, 257), (2, 2, 48, 3), (300, 3, 64, 1), (1, 33000, 16, 2), (300, 1, 2047, 1), (2100, 1, 1030, 1), (17, 1, 4096, 1),
    (4, 49, 768, 32), (3, 500, 64, 8), (1, 20000, 24, 3), (2, 2500, 256, 32),
    # many small images, several a workgroup
    (2101, 1, 64, 4), (4099, 1, 24, 3), (3001, 2, 40, 5), (1025, 9, 64, 8), (1537, 4, 256, 32), (5003, 1, 6, 3), (1300, 7, 10, 2), (1027, 33, 16, 1),
    # groups of 4 and 2 values at a time
    (3, 500, 36, 3), (2, 1700, 30, 3), (1100, 3, 24, 4), (1, 9001, 84, 7), (2, 300, 1036, 1), (6, 49, 770, 77),
]


def _norm_inputs(dtype, B, N, C, offset=0.5, seed=0):
    g = np.random.default_rng(seed + B * 7919 + N * 31 + C)
    a = {"x": g.normal(size=(B, N, C)) * (0.5 + g.random(C)) + offset * g.normal(size=C), "gamma": 1 + 0.3 * g.normal(size=C), "beta": 0.3 * g.normal(size=C),
         "dout": g.normal(size=(B, N, C))}
    return {k: _stored(v, dtype) for k, v in a.items()}


def _sum_error(n):
    """Of a sum of n terms, relative to the sum of their absolute values: lanes add at most n / 64 + 32 terms one after another
    before the partial sums are added pairwise or in short rows (64 more)."""
    return U * (n / 64 + 96)


def _norm_fwd_bounds(v, G, eps, name, affine, dtype):
    x = v["x"]
    B, N, C = x.shape
    gamma, beta = (v["gamma"], v["beta"]) if affine else (None, None)
    out, mean, rstd = dense.norm_fwd(x, gamma, beta, G, eps, name)
    n = N * C // G
    e = _sum_error(n)
    xg = x.reshape(B, N, G, C // G)
    dm = e * np.abs(xg).mean(axis=(1, 3)) + U * np.abs(mean)
    var = 1.0 / rstd ** 2
    rel = 0.5 * (e + 4 * U + dm ** 2 / var + 2 * U * 8) + 4 * U  # of rstd: variance, its square root and reciprocal
    dr = rel * rstd
    wide = lambda t: np.broadcast_to(t[:, None, :, None], xg.shape).reshape(x.shape)
    ag = np.abs(gamma) if affine else 1.0
    xhat = np.abs(x - wide(mean)) * wide(rstd)
    dz = ag * (wide(dm * rstd) * (1 + 1e-3) + xhat * (wide(rel) + 4 * U)) + (U * np.abs(beta) if affine else 0)
    z = xhat * ag + (np.abs(beta) if affine else 0)
    d = SLOPE * dz + U * z + (0 if name == "none" else 8 * U * (1 + z))
    return out, mean, rstd, d + HALF[dtype] * (np.abs(out) + d), dm, dr


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C,G", NORM)
def test_norm_forward(dtype, B, N, C, G):
    name = ["none", "silu", "relu", "gelu"][(B + N + C) % 4]
    affine = (B + C) % 4 != 0
    d = _norm_inputs(dtype, B, N, C)
    out, mean, rstd, tol, dm, dr = _norm_fwd_bounds({k: a[1] for k, a in d.items()}, G, 1e-5, name, affine, dtype)
    go, gm, gr = Guarded((B, N, C), TYPES[dtype]), Guarded((B, G), torch.float32), Guarded((B, G), torch.float32)
    aff.affmae_norm_fwd(d["x"][0], d["gamma"][0] if affine else None, d["beta"][0] if affine else None, G, 1e-5, act=name, out=go.t, mean=gm.t, rstd=gr.t)
    _close(gm.t, mean, dm, "mean")
    _close(gr.t, rstd, dr, "rstd")
    _close(go.t, out, tol, "out")
    for o in (go, gm, gr):
        o.check()


def _norm_bwd_bounds(v, mean, rstd, G, name, affine, dtype):
    x, dout = v["x"], v["dout"]
    B, N, C = x.shape
    gamma, beta = (v["gamma"], v["beta"]) if affine else (None, None)
    ref = dense.norm_bwd(x, gamma, beta, mean, rstd, dout, G, name)
    ag = np.abs(gamma) if affine else 1.0
    g4 = lambda t: t.reshape(B, N, G, C // G)
    wide = lambda t: np.broadcast_to(t[:, None, :, None], (B, N, G, C // G)).reshape(x.shape)
    xhat = np.abs(x - wide(mean)) * wide(rstd)
    z = xhat * ag + (np.abs(beta) if affine else 0)
    dz = np.abs(dout * dense.slope((x - wide(mean)) * wide(rstd) * (gamma if affine else 1.0) + (beta if affine else 0.0), name))
    edz = 2 * U * dz + (0 if name == "none" else 8 * U * np.abs(dout) * (1 + z))  # |slope'| <= 1 times the error 4 U z of z is in it
    if name == "relu":  # next to the corner the slope may be either
        edz = edz + np.abs(dout) * (np.abs((x - wide(mean)) * wide(rstd) * (gamma if affine else 1.0) + (beta if affine else 0.0)) <= 8 * U * (1 + z))
    dh, edh = dz * ag, (edz + U * dz) * ag
    n = N * C // G
    e = _sum_error(n)
    s1, es1 = g4(dh).mean(axis=(1, 3)), g4(edh).mean(axis=(1, 3)) + (e + 2 * U) * g4(dh).mean(axis=(1, 3))
    s2 = g4(dh * xhat).mean(axis=(1, 3))
    es2 = g4(edh * xhat + 3 * U * dh * xhat).mean(axis=(1, 3)) + (e + 2 * U) * s2
    d = wide(rstd) * (edh + wide(es1) + xhat * wide(es2) + 4 * U * (dh + wide(s1) + xhat * wide(s2)))
    rows = _sum_error(B * N)
    bounds = {"dx": d + HALF[dtype] * (np.abs(ref["dx"]) + d),
              "dgamma": (edz * xhat + 3 * U * dz * xhat).sum((0, 1)) + rows * (dz * xhat).sum((0, 1)),
              "dbeta": edz.sum((0, 1)) + rows * dz.sum((0, 1))}
    return ref, bounds


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C,G", NORM)
def test_norm_backward(dtype, B, N, C, G):
    name = ["silu", "none", "gelu", "relu"][(B + N + C) % 4]
    affine = (B + N) % 4 != 0
    d = _norm_inputs(dtype, B, N, C, seed=1)
    v = {k: a[1] for k, a in d.items()}
    _, mean, rstd = dense.norm_fwd(v["x"], v["gamma"], v["beta"], G, 1e-5)
    (tm, mean), (tr, rstd) = _stored(mean, "f32"), _stored(rstd, "f32")
    ref, bounds = _norm_bwd_bounds(v, mean, rstd, G, name, affine, dtype)
    g = {"dx": Guarded((B, N, C), TYPES[dtype])}
    if affine:
        g.update(dgamma=Guarded((C,), torch.float32), dbeta=Guarded((C,), torch.float32))
    args = (d["x"][0], d["gamma"][0] if affine else None, d["beta"][0] if affine else None, tm, tr, d["dout"][0], G)
    aff.affmae_norm_bwd(*args, act=name, grads={k: o.t for k, o in g.items()})
    for k in g:
        _close(g[k].t, ref[k], bounds[k], k)
        g[k].check()
    again = aff.affmae_norm_bwd(*args, act=name)
    assert set(again) == set(g) and all(torch.equal(again[k], g[k].t) for k in g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 4])
@pytest.mark.parametrize("B,N,C,G", [(40, 1, 64, 1), (2, 90, 64, 4)])
def test_norm_of_tensors_off_their_alignment(dtype, shift, B, N, C, G):
    d = _norm_inputs(dtype, B, N, C, seed=2)
    v = {k: a[1] for k, a in d.items()}
    s = {k: _shifted(a[0], shift) for k, a in d.items()}
    out, mean, rstd, tol, dm, dr = _norm_fwd_bounds(v, G, 1e-5, "silu", True, dtype)
    go = Guarded((B, N, C), TYPES[dtype], shift)
    _, m, r = aff.affmae_norm_fwd(s["x"], s["gamma"], s["beta"], G, act="silu", out=go.t)
    _close(go.t, out, tol, "out")
    go.check()
    ref, bounds = _norm_bwd_bounds(v, m.double().cpu().numpy(), r.double().cpu().numpy(), G, "silu", True, dtype)
    gx = Guarded((B, N, C), TYPES[dtype], shift)
    got = aff.affmae_norm_bwd(s["x"], s["gamma"], s["beta"], _shifted(m, 1), _shifted(r, 1), s["dout"], G, act="silu", grads={"dx": gx.t})
    gx.check()
    for k in got:
        _close(got[k], ref[k], bounds[k], k)


@pytest.mark.parametrize("B,N,C,G", [(20, 1, 256, 1), (2, 3000, 32, 4), (3, 1, 6000, 1)])
def test_norm_of_values_far_from_zero_and_of_outliers(B, N, C, G):
    """Offsets of 1000 spreads, and one value of 1e6 spreads at the place that a shifted sum would take its shift from."""
    d = _norm_inputs("f32", B, N, C, seed=3)
    for far in (True, False):
        x = d["x"][1] + 1000.0 if far else d["x"][1].copy()
        if not far:
            x[:, 0, 0] = 1e6
        t, x = _stored(x, "f32")
        v = {"x": x, "gamma": d["gamma"][1], "beta": d["beta"][1]}
        out, mean, rstd, tol, dm, dr = _norm_fwd_bounds(v, G, 1e-5, "none", True, "f32")
        o, m, r = aff.affmae_norm_fwd(t, d["gamma"][0], d["beta"][0], G)
        _close(m, mean, dm, "mean")
        _close(r, rstd, dr, "rstd")
        _close(o, out, tol, "out")


def test_norm_of_constant_values():
    """No spread at all: rstd = eps^-1/2, the result is beta; the gradients stay finite."""
    for B, N, C, G in ((4, 1, 64, 1), (2, 500, 24, 3)):
        x = torch.full((B, N, C), 3.0, device="cuda")
        gamma, beta = torch.full((C,), 2.0, device="cuda"), torch.linspace(-1, 1, C, device="cuda")
        out, mean, rstd = aff.affmae_norm_fwd(x, gamma, beta, G, 1e-5)
        assert bool((mean == 3).all()) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)
        assert torch.equal(out, beta.expand_as(out))
        g = aff.affmae_norm_bwd(x, gamma, beta, mean, rstd, torch.ones_like(x), G)
        assert all(bool(torch.isfinite(t).all()) for t in g.values())


@pytest.mark.parametrize("B,N", [(3, 40), (3000, 2)])
def test_norm_keeps_what_is_not_finite_in_its_group(B, N):
    x = torch.randn(B, N, 32, device="cuda")
    x[1, N // 2, 9] = float("nan")
    out, mean, rstd = aff.affmae_norm_fwd(x, None, None, 4)
    bad = torch.zeros(B, 4, dtype=torch.bool, device="cuda")
    bad[1, 1] = True
    assert torch.equal(torch.isnan(mean), bad) and torch.equal(torch.isnan(rstd), bad)
    wide = bad[:, None, :, None].expand(B, N, 4, 8).reshape(B, N, 32)
    assert torch.equal(torch.isnan(out), wide)
    good = torch.randn(B, 4, device="cuda").abs() + 0.5
    dx = aff.affmae_norm_bwd(torch.nan_to_num(x), None, None, torch.where(bad, mean, good), good, torch.ones_like(x), 4)["dx"]
    assert torch.equal(torch.isnan(dx), wide)


# --------------------------------------------------------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 4, 8, 1000, 4099, 65536, 100008])
@pytest.mark.parametrize("p", [0.0, 1e-9, 0.1, 0.999])
def test_dropout(dtype, n, p):
    g = np.random.default_rng(n)
    (x, xv), (r, rv) = _stored(g.normal(size=n), dtype), _stored(g.normal(size=n), dtype)
    rng = _rng() if p else None
    ref = dense.drop(xv, p, SEED)
    tol = 2 * U * np.abs(ref)
    for residual in (False, True):
        go = Guarded((n,), TYPES[dtype])
        aff.affmae_dropout_fwd(x, p, rng, residual=r if residual else None, out=go.t)
        full = rv + ref if residual else ref
        t = tol + (U * np.abs(full) if residual else 0)
        _close(go.t, full, t + HALF[dtype] * (np.abs(full) + t), "out")
        go.check()
        if p and not residual:
            assert np.array_equal(go.t.cpu().float().numpy() == 0, ~dense.keep((n,), p, *SEED))
    dx = aff.affmae_dropout_bwd(x, p, rng)
    assert torch.equal(dx, aff.affmae_dropout_fwd(x, p, rng))
    # in place, and off the alignment
    y = x.clone()
    assert aff.affmae_dropout_fwd(y, p, rng, out=y) is y and torch.equal(y, dx)
    for shift in (1, 2):
        go = Guarded((n,), TYPES[dtype], shift)
        aff.affmae_dropout_bwd(_shifted(x, shift), p, rng, dx=go.t)
        assert torch.equal(go.t, dx)
        go.check()


@pytest.mark.parametrize("seed,call", [(0, 0), (-1, -1), (2 ** 63 - 1, -2 ** 63), (1 << 40, 1 << 33)])
def test_dropout_takes_all_bits_of_seed_and_call_number(seed, call):
    x = torch.ones(1000, device="cuda")
    got = aff.affmae_dropout_fwd(x, 0.5, torch.tensor([seed, call], dtype=torch.int64, device="cuda"))
    assert np.array_equal(got.cpu().numpy() != 0, dense.keep((1000,), 0.5, seed, call))


def test_dropout_replaces_what_is_not_finite():
    n = 4096
    keep = torch.from_numpy(dense.keep((n,), 0.5, *SEED)).cuda()
    for bad in (float("inf"), float("nan")):
        got = aff.affmae_dropout_fwd(torch.full((n,), bad, device="cuda"), 0.5, _rng())
        assert bool((got[~keep] == 0).all()) and not bool(torch.isfinite(got[keep]).any())


def test_dropout_of_more_than_2_32_elements():
    """Places beyond 32 bits: the last elements of a tensor of 2^32 + 1003."""
    n = 2 ** 32 + 1003
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    aff.affmae_dropout_fwd(x, 0.5, _rng(), out=x)
    first = 2 ** 32 - 1000
    words = dense.philox(*SEED, first // 4, -(-(n - first) // 4)).reshape(-1)[:n - first]
    assert np.array_equal(x[first:].float().cpu().numpy() != 0, words >= np.uint64(2 ** 31))
    words = dense.philox(*SEED, 0, 250).reshape(-1)
    assert np.array_equal(x[:1000].float().cpu().numpy() != 0, words >= np.uint64(2 ** 31))


def test_linear_beyond_2_31_values():
    """Tensors of more than 2^31 values.  Whole numbers of at most two digits: every sum is exact, whatever its order."""
    rows, cin, cout = 33_600_005, 64, 72
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    small = lambda *shape: torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8).bfloat16()
    x, w, dout = small(rows, cin), small(cout, cin), small(rows, cout)
    out, _ = aff.affmae_linear_fwd(x, w)
    for lo in (0, rows // 2, rows - 4099):
        assert torch.equal(out[lo:lo + 4099].float(), x[lo:lo + 4099].float() @ w.float().t())
    del out
    got = aff.affmae_linear_bwd(x, w, dout, dout, act="relu")  # dz: dout where it is 1
    for lo in (0, rows // 2, rows - 4099):
        assert torch.equal(got["dx"][lo:lo + 4099].float(), (dout[lo:lo + 4099] > 0).float() @ w.float())
    dw, db = torch.zeros(cout, cin, dtype=torch.float64, device="cuda"), torch.zeros(cout, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 1 << 22):
        z = (dout[lo:lo + (1 << 22)] > 0).double()
        dw += z.t().contiguous() @ x[lo:lo + (1 << 22)].double()
        db += z.sum(0)
    assert float(dw.abs().max()) < 2 ** 24 and float(db.max()) < 2 ** 24
    assert torch.equal(got["dweight"], dw.bfloat16()) and torch.equal(got["dbias"], db.bfloat16())


def test_norm_beyond_2_31_values():
    """-1, 1, -1, ... in tensors of more than 2^31 values: mean 0 and variance 1, exactly."""
    for B, N, C, G in ((2, 9_000_005, 128, 4), (16_777_215, 1, 136, 1)):
        x = torch.ones(B, N, C, dtype=torch.bfloat16, device="cuda")
        x[..., ::2] = -1
        gamma, beta = torch.full((C,), 3.0, device="cuda").bfloat16(), torch.zeros(C, device="cuda").bfloat16()
        out, mean, rstd = aff.affmae_norm_fwd(x, gamma, beta, G, eps=1e-5)
        assert bool((mean == 0).all()) and bool(((rstd - (1 + 1e-5) ** -0.5).abs() < 4 * U).all())
        want = x.view(-1)[:C] * 3
        for lo in (0, B * N // 2, B * N - 5000):
            assert torch.equal(out.view(-1, C)[lo:lo + 5000], want.expand(5000, C))
        del out
        # dout = x: dh = 3 x = 3 xhat (up to eps), so dx is 3 x (1 - 1 / (1 + eps)) rstd; dgamma counts the tokens, dbeta too, with signs
        got = aff.affmae_norm_bwd(x, gamma, beta, mean, rstd, x, G)
        for lo in (0, B * N // 2, B * N - 5000):
            assert float(got["dx"].view(-1, C)[lo:lo + 5000].float().abs().max()) < 1e-4
        tokens = float(B * N)
        assert float((got["dgamma"].double() / tokens - (1 + 1e-5) ** -0.5).abs().max()) < _sum_error(B * N)
        assert float((got["dbeta"].double() / tokens - x.view(-1)[:C].double()).abs().max()) < _sum_error(B * N)
        del got, x


def test_norm_of_as_many_tokens_as_there_may_be():
    """One image of 2^31 - 2^16 tokens of one channel, -1, 1, -1, ...: mean 0 and variance 1, exactly."""
    N = 2 ** 31 - 2 ** 16
    x = torch.ones(1, N, 1, dtype=torch.bfloat16, device="cuda")
    x[:, ::2] = -1
    gamma, beta = torch.full((1,), 3.0, device="cuda").bfloat16(), torch.zeros(1, device="cuda").bfloat16()
    out, mean, rstd = aff.affmae_norm_fwd(x, gamma, beta, 1, eps=1e-5)
    assert float(mean) == 0 and abs(float(rstd) - (1 + 1e-5) ** -0.5) < 4 * U
    for lo in (0, N // 2, N - 5000):
        assert torch.equal(out[:, lo:lo + 5000], x[:, lo:lo + 5000] * 3)
    got = aff.affmae_norm_bwd(x, gamma, beta, mean, rstd, x, 1, grads={"dx": out})
    assert float(got["dx"][:, -5000:].float().abs().max()) < 1e-4
    assert abs(float(got["dgamma"]) / N - (1 + 1e-5) ** -0.5) < _sum_error(N) and abs(float(got["dbeta"])) <= _sum_error(N) * N


# -------------------------------------------------------------------------------------------------------------- refusals

def test_binding_refuses():
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    for bad in (lambda: aff.affmae_linear_fwd(x.t(), w), lambda: aff.affmae_linear_fwd(x, w.t()), lambda: aff.affmae_linear_fwd(x, w[:, :4]),
                lambda: aff.affmae_linear_fwd(x, w.bfloat16()), lambda: aff.affmae_linear_fwd(x, w, w[:, 0]), lambda: aff.affmae_linear_fwd(x, w, x[0]),
                lambda: aff.affmae_linear_fwd(x, w, act="tanh"), lambda: aff.affmae_linear_fwd(x, w, p=0.5),
                lambda: aff.affmae_linear_fwd(x, w, p=0.5, rng=torch.zeros(2, device="cuda")), lambda: aff.affmae_linear_fwd(x, w, residual=x),
                lambda: aff.affmae_linear_fwd(x, w, bias=torch.zeros(6)), lambda: aff.affmae_linear_fwd(x, w, p=0.5, rng=torch.zeros(2, dtype=torch.int64)),
                lambda: aff.affmae_linear_bwd(x, w, x), lambda: aff.affmae_linear_bwd(None, w, torch.zeros(4, 6, device="cuda")),
                lambda: aff.affmae_linear_bwd(x, w, torch.zeros(4, 6, device="cuda"), act="gelu"),
                lambda: aff.affmae_norm_fwd(x, None, None), lambda: aff.affmae_norm_fwd(x[None], w[0], None), lambda: aff.affmae_norm_fwd(x[None], w[:, 0], w[:, 0]),
                lambda: aff.affmae_norm_fwd(x[None].transpose(1, 2), None, None), lambda: aff.affmae_norm_bwd(x[None], None, None, x, x, x[None], 2),
                lambda: aff.affmae_dropout_fwd(x.t(), 0.1, _rng()), lambda: aff.affmae_dropout_fwd(x, 0.1), lambda: aff.affmae_dropout_bwd(x, 0.1, _rng()[:1])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: aff.affmae_linear_fwd(x[:0], w), lambda: aff.affmae_linear_fwd(x, w, p=1.0, rng=_rng()), lambda: aff.affmae_norm_fwd(x[None], None, None, 3),
                lambda: aff.affmae_norm_fwd(x[None], None, None, 2, eps=0.0), lambda: aff.affmae_dropout_fwd(x[:0], 0.1, _rng()),
                lambda: aff.affmae_linear_bwd(x, w, torch.zeros(4, 6, device="cuda"), torch.zeros(4, 6, device="cuda"), act="relu",
                                              workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(aff.AffmaeError):
            bad()


# ---------------------------------------------------------------------------------------------- together, graphs, streams

def _block(t, nbr, H, scale, p, rng):
    """A pre-norm block over x [B,N,C] and its gradients: norm, q/k/v, neighbourhood attention, product + dropout + residual; norm,
    product + activation, product + dropout + residual."""
    B, N, C = t["x"].shape
    x = t["x"]
    one = lambda v: v.view(B * N, 1, C)
    n1, m1, r1 = aff.affmae_norm_fwd(one(x), t["g1"], t["b1"])
    n1 = n1.view(B, N, C)
    q, k, v = (aff.affmae_linear_fwd(n1, t["w" + c], t["c" + c])[0].view(B, N, H, C // H) for c in "qkv")
    att, lse = aff.affmae_pla_fwd(q, k, v, None, nbr, scale)
    h, _ = aff.affmae_linear_fwd(att.view(B, N, C), t["wo"], t["co"], residual=x, p=p, rng=rng[0])
    n2, m2, r2 = aff.affmae_norm_fwd(one(h), t["g2"], t["b2"])
    n2 = n2.view(B, N, C)
    u, pre = aff.affmae_linear_fwd(n2, t["wu"], t["cu"], act="gelu", want_pre=True)
    y, _ = aff.affmae_linear_fwd(u, t["wd"], t["cd"], residual=h, p=p, rng=rng[1])
    g = {}
    down = aff.affmae_linear_bwd(u, t["wd"], t["dy"], p=p, rng=rng[1])
    up = aff.affmae_linear_bwd(n2, t["wu"], down["dx"], pre, act="gelu")
    norm2 = aff.affmae_norm_bwd(one(h), t["g2"], t["b2"], m2, r2, one(up["dx"]))
    dh = t["dy"] + norm2["dx"].view(B, N, C)
    o = aff.affmae_linear_bwd(att.view(B, N, C), t["wo"], dh, p=p, rng=rng[0])
    a = aff.affmae_pla_bwd(q, k, v, None, nbr, att, lse, o["dx"].view(B, N, H, C // H), scale, want_dbias=False)
    dn1 = 0
    for c in "qkv":
        gc = aff.affmae_linear_bwd(n1, t["w" + c], a["d" + c].view(B, N, C))
        dn1 = dn1 + gc["dx"]
        g["w" + c], g["c" + c] = gc["dweight"], gc["dbias"]
    norm1 = aff.affmae_norm_bwd(one(x), t["g1"], t["b1"], m1, r1, one(dn1))
    g.update(x=dh + norm1["dx"].view(B, N, C), g1=norm1["dgamma"], b1=norm1["dbeta"], g2=norm2["dgamma"], b2=norm2["dbeta"], wo=o["dweight"], co=o["dbias"],
             wu=up["dweight"], cu=up["dbias"], wd=down["dweight"], cd=down["dbias"])
    return y, g, a["dk"]


def _block_reference(v, nbr, H, scale, p, rng):
    B, N, C = v["x"].shape
    one = lambda a: a.reshape(B * N, 1, C)
    flat = lambda a: a.reshape(B * N, -1)
    x = v["x"]
    n1, m1, r1 = dense.norm_fwd(one(x), v["g1"], v["b1"], 1, 1e-5)
    q, k, w = (dense.linear_fwd(flat(n1), v["w" + c], v["c" + c])[0].reshape(B, N, H, C // H) for c in "qkv")
    att, _ = oracle.pla_fwd(q, k, w, None, nbr, scale)
    h = dense.linear_fwd(flat(att), v["wo"], v["co"], flat(x), "none", p, rng[0])[0]
    n2, m2, r2 = dense.norm_fwd(one(h), v["g2"], v["b2"], 1, 1e-5)
    u, pre = dense.linear_fwd(flat(n2), v["wu"], v["cu"], None, "gelu")
    y = dense.linear_fwd(u, v["wd"], v["cd"], h, "none", p, rng[1])[0]
    dy = flat(v["dy"])
    down = dense.linear_bwd(u, v["wd"], dy, None, "none", p, rng[1])
    up = dense.linear_bwd(flat(n2), v["wu"], down["dx"], pre, "gelu")
    norm2 = dense.norm_bwd(one(h), v["g2"], v["b2"], m2, r2, one(up["dx"]), 1)
    dh = dy + flat(norm2["dx"])
    o = dense.linear_bwd(flat(att), v["wo"], dh, None, "none", p, rng[0])
    a = oracle.pla_bwd(q, k, w, None, nbr, o["dx"].reshape(B, N, H, C // H), scale)
    g, dn1 = {}, 0
    for c in "qkv":
        gc = dense.linear_bwd(flat(n1), v["w" + c], flat(a["d" + c]))
        dn1 = dn1 + gc["dx"]
        g["w" + c], g["c" + c] = gc["dweight"], gc["dbias"]
    norm1 = dense.norm_bwd(one(x), v["g1"], v["b1"], m1, r1, one(dn1), 1)
    g.update(x=(dh + flat(norm1["dx"])).reshape(x.shape), g1=norm1["dgamma"], b1=norm1["dbeta"], g2=norm2["dgamma"], b2=norm2["dbeta"], wo=o["dweight"],
             co=o["dbias"], wu=up["dweight"], cu=up["dbias"], wd=down["dweight"], cd=down["dbias"])
    return y.reshape(x.shape), g


def _block_inputs(dtype, B, N, C, seed=0):
    g = np.random.default_rng(seed)
    a = {"x": g.normal(size=(B, N, C)), "dy": g.normal(size=(B, N, C))}
    for c in "qkvo":
        a["w" + c], a["c" + c] = g.normal(size=(C, C)) / np.sqrt(C), 0.1 * g.normal(size=C)
    a["wu"], a["cu"], a["wd"], a["cd"] = g.normal(size=(3 * C, C)) / np.sqrt(C), 0.1 * g.normal(size=3 * C), g.normal(size=(C, 3 * C)) / np.sqrt(3 * C), 0.1 * g.normal(size=C)
    for i in "12":
        a["g" + i], a["b" + i] = 1 + 0.2 * g.normal(size=C), 0.2 * g.normal(size=C)
    d = {k: _stored(v, dtype) for k, v in a.items()}
    nbr = np.stack([np.stack([g.permutation(N)[:9] for _ in range(N)]) for _ in range(B)]).astype(np.int32)
    return {k: v[0] for k, v in d.items()}, {k: v[1] for k, v in d.items()}, nbr


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 2e-1)])
def test_block_forward_and_backward(dtype, tol):
    """Ten operators one after another.  Each is held to max|err| / max|ref| <= 1e-5 (fp32) / 2e-2 (bf16) by itself; of ten in a row
    with gains about 1 the errors add up to ten times that."""
    B, N, C, H, p = 2, 150, 64, 2, 0.2
    t, v, nbr = _block_inputs(dtype, B, N, C)
    rng = torch.tensor([[5, 1], [5, 2]], dtype=torch.int64, device="cuda")
    y, g, _ = _block(t, torch.from_numpy(nbr).cuda(), H, 0.18, p, rng)
    ry, rg = _block_reference(v, nbr, H, 0.18, p, [(5, 1), (5, 2)])
    errs = {"y": np.abs(y.double().cpu().numpy() - ry).max() / np.abs(ry).max()}
    for k in rg:
        errs[k] = np.abs(g[k].double().cpu().numpy() - rg[k]).max() / max(np.abs(rg[k]).max(), 1e-30)
    # (the key's bias moves all logits of a query alike: its gradient is 0, up to the errors of the sum of |terms|)
    ck = np.abs(rg["cq"]).max()
    errs["ck"] = np.abs(g["ck"].double().cpu().numpy() - rg["ck"]).max() / ck
    assert set(g) == set(rg) and max(errs.values()) <= tol, errs


def test_block_replayed_from_a_graph_on_another_stream():
    """One graph of a whole block's forward and backward, with the generator's call numbers advanced on the device between the replays:
    every replay equals the eager result, bit by bit where sums have a fixed order."""
    B, N, C, H, p = 2, 200, 64, 2, 0.3
    t, v, nbr = _block_inputs("bf16", B, N, C, 7)
    nbr = torch.from_numpy(nbr).cuda()
    rng = torch.tensor([[5, 1], [5, 2]], dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _block(t, nbr, H, 0.18, p, rng)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y, g, _ = _block(t, nbr, H, 0.18, p, rng)
    seen = []
    for rep in range(4):
        rng[:, 1] += 2
        t["x"].add_(0.125)
        ey, eg, edk = _block(t, nbr, H, 0.18, p, rng)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ey), f"replay {rep}"
        for k in ("wd", "cd", "wu", "cu", "g2", "b2"):  # in front of the attention's backward, whose sums may change in the last bits
            assert torch.equal(g[k], eg[k]), f"replay {rep}: {k}"
        for k in eg:
            atol = 2e-2 * float(eg[k].float().abs().max())
            if k == "ck":
                # The key's bias moves all logits of a query alike: its gradient is 0, and what is left of the sum over 400 tokens is
                # their rounding.  dk is added up in an order that changes by 2^-22 of the terms or so, and a value as near to the middle
                # of a step of bf16 as that (one in 2^13) is rounded the other way: by 2^-7 of the value.  Four in a channel's 400 are a bound
                # that 64 channels x 4 replays exceed once in 1e6 runs (Poisson with mean 400 / 2^13 = 0.05: 256 x 0.05^5 / 5! = 7e-7).
                atol = 4 * 2.0 ** -7 * float(edk.float().abs().max())
            assert torch.allclose(g[k].float(), eg[k].float(), rtol=2e-2, atol=atol), f"replay {rep}: {k}"
        seen.append(y.clone())
    assert all(not torch.equal(a, b) for a, b in zip(seen, seen[1:]))


def test_large_products_replayed_from_a_graph():
    """Tiles of more than 64 KB of LDS, k split over workgroups, statistics of several launches: replays with new inputs, eager work of the
    same calls between them."""
    rows, cin, cout = 16400, 776, 2312
    x, w, dout, pre = (torch.randn(*s, device="cuda").bfloat16() for s in ((rows, cin), (cout, cin), (rows, cout), (rows, cout)))
    nx, nd, gamma, beta = (torch.randn(*s, device="cuda") for s in ((2, 9000, 48), (2, 9000, 48), (48,), (48,)))
    rng = _rng()

    def run():
        out, _ = aff.affmae_linear_fwd(x, w, act="silu", p=0.5, rng=rng)
        g = aff.affmae_linear_bwd(x, w, dout, pre, act="silu", p=0.5, rng=rng)
        y, m, r = aff.affmae_norm_fwd(nx, gamma, beta, 6, act="gelu")
        h = aff.affmae_norm_bwd(nx, gamma, beta, m, r, nd, 6, act="gelu")
        return [out, y, m, r, aff.affmae_dropout_fwd(nx, 0.3, rng), *g.values(), *h.values()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run()
    for rep in range(3):
        rng[1] += 1
        x.mul_(0.5)
        nx.add_(1.0)
        ref = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), f"replay {rep}"


def test_copies_and_small_images_replayed_from_a_graph():
    """Gradients that write copies of odd rows, and norms of several images a workgroup, forward and backward."""
    rows, cin, cout = 3001, 1281, 1283
    x, w, dout = (torch.randn(*s, device="cuda").bfloat16() for s in ((rows, cin), (cout, cin), (rows, cout)))
    nx, nd, gamma, beta = (torch.randn(*s, device="cuda").bfloat16() for s in ((3001, 3, 64), (3001, 3, 64), (64,), (64,)))

    def run():
        g = aff.affmae_linear_bwd(x, w, dout)
        y, m, r = aff.affmae_norm_fwd(nx, gamma, beta, 4, act="silu")
        h = aff.affmae_norm_bwd(nx, gamma, beta, m, r, nd, 4, act="silu")
        return [y, m, r, *g.values(), *h.values()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run()
    for rep in range(3):
        x.mul_(0.5)
        nx.add_(1.0)
        ref = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), f"replay {rep}"


def test_calls_on_two_streams_at_once():
    d = _linear_inputs("bf16", 20000, 64, 192, 8)
    x, w, b, dout, pre = (d[k][0] for k in ("x", "w", "b", "dout", "pre"))
    n = _norm_inputs("bf16", 4, 5000, 64, seed=9)
    nx, nd = n["x"][0], n["dout"][0]

    def run():
        out, _ = aff.affmae_linear_fwd(x, w, b, act="gelu", p=0.1, rng=rng)
        g = aff.affmae_linear_bwd(x, w, dout, pre, act="gelu", p=0.1, rng=rng)
        y, m, r = aff.affmae_norm_fwd(nx, n["gamma"][0], n["beta"][0], 8)
        h = aff.affmae_norm_bwd(nx, n["gamma"][0], n["beta"][0], m, r, nd, 8)
        return [out, y, m, r, *g.values(), *h.values()]

    rng = _rng()
    ref = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                results.append(run())
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
