"""GPU parity of attention between all tokens and of rotary positions against the plain 64-bit implementations (oracle/attn.py) on the same
stored values, value by value.

Bounds (oracle/attn.py works them out beside the values): U is half a step of fp32 and half(dtype) half a step of the storage type,
relative to the value.  A sum of n terms in fp32 is off by at most 2 U (n + 6 to 16) times the sum of the terms' absolute values, whatever the
order (2 U instead of U: matrix instructions may truncate).  A score is off by its product's bound, 8 U of the cap and 8 U of the distance's
term; p by the score's error, the largest one of its row (through the sum), the sum's and the exponential's; bf16 rounds p and dS once more
as operands of the products."""
import numpy as np
import pytest
import torch

import paper_2602_16249_amd as aff
from oracle import attn as oa

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -24


def _stored(a, dtype):
    """A device tensor of the storage type, and the values that it holds."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPES[dtype])
    return t.cuda(), t.double().numpy()


def _close(got, ref, tol, what):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, what
    same = got == ref  # (infinities)
    with np.errstate(invalid="ignore"):
        over = ~(same | (np.abs(got - ref) <= tol))
    if over.any():
        i = tuple(int(v) for v in np.argwhere(over)[0])
        raise AssertionError(f"{what}: {int(over.sum())} of {over.size} off, first at {i}: {got[i]} for {ref[i]}, bound {np.broadcast_to(tol, ref.shape)[i]}")


class Guarded:
    """An output inside a larger buffer whose other elements have to stay as they were."""

    def __init__(self, shape, dtype):
        n = int(np.prod(shape))
        self.n, self.lo = n, 128
        self.buf = torch.full((n + 256,), 77.0, dtype=dtype, device="cuda")
        self.t = self.buf[self.lo:self.lo + n].view(shape)

    def check(self):
        assert bool((self.buf[:self.lo] == 77).all()) and bool((self.buf[self.lo + self.n:] == 77).all()), "written outside"


def _docs(g, B, N, kind):
    """Images of the tokens: in runs of uneven length with padding between them, or in any order."""
    if kind == "runs":
        ids = np.sort(g.integers(0, max(2, N // 23), (B, N)), axis=1)
        ids[g.random((B, N)) < 0.08] = -1
        ids[:, N - N // 9:] = -1 - g.integers(0, 5)
    else:
        ids = g.integers(-1, 4, (B, N))
    return ids.astype(np.int32)


def _case(dtype, B, Nq, Nk, H, Hk, d, cap=0.0, distance=False, docs=None, seed=0, poison=True):
    """Device tensors and the values that they hold; padding holds NaN on the device."""
    g = np.random.default_rng(seed + 7919 * Nq + 31 * Nk + H + d)
    dev, val = {}, {}
    for n, shape in (("q", (B, Nq, H, d)), ("k", (B, Nk, Hk, d)), ("v", (B, Nk, Hk, d)), ("dout", (B, Nq, H, d))):
        dev[n], val[n] = _stored(g.normal(size=shape), dtype)
    terms, tval = {}, {}
    if distance:
        same = Nq == Nk
        k_xy = g.uniform(0, 100, (B, Nk, 2))
        for n, x in (("k_xy", k_xy), ("q_xy", k_xy if same else g.uniform(0, 100, (B, Nq, 2))), ("slope", g.uniform(-0.01, 0.08, H))):
            terms[n], tval[n] = _stored(x, "f32")
    if docs:
        tval["k_doc"] = _docs(g, B, Nk, docs)
        tval["q_doc"] = tval["k_doc"] if Nq == Nk else _docs(g, B, Nq, docs)
        terms.update({n: torch.from_numpy(tval[n]).cuda() for n in ("q_doc", "k_doc")})
        if poison:
            for n, doc in (("q", "q_doc"), ("dout", "q_doc"), ("k", "k_doc"), ("v", "k_doc")):
                dev[n][terms[doc] < 0] = float("nan")
            if distance:
                terms["q_xy"] = terms["q_xy"].clone()
                terms["q_xy"][terms["q_doc"] < 0] = float("nan")
                terms["k_xy"][terms["k_doc"] < 0] = float("inf")
    return dev, val, terms, tval


def _check(dtype, shape, scale=None, cap=0.0, distance=False, docs=None, seed=0):
    B, Nq, Nk, H, Hk, d = shape
    scale = d ** -0.5 if scale is None else scale
    dev, val, terms, tval = _case(dtype, *shape, cap=cap, distance=distance, docs=docs, seed=seed)
    o, l = Guarded((B, Nq, H, d), TYPES[dtype]), Guarded((B, Nq, H), torch.float32)
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], scale, cap, out=o.t, lse=l.t, **terms)
    g = {n: Guarded(dev[n[1:]].shape, TYPES[dtype]) for n in ("dq", "dk", "dv")}
    if distance:
        g["dslope"] = Guarded((H,), torch.float32)
    aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], scale, cap, grads={n: x.t for n, x in g.items()}, **terms)
    given = out.double().cpu().numpy()
    scale = float(np.float32(scale))
    ref = oa.attn(val["q"], val["k"], val["v"], scale, float(np.float32(cap)), dout=val["dout"], half=HALF[dtype], given=given, **tval)
    _close(out, *ref["out"], "out")
    _close(lse, *ref["lse"], "lse")
    for n in g:
        _close(g[n].t, *ref[n], n)
    for x in (o, l, *g.values()):
        x.check()
    if docs:  # padding gets zeros
        for n, doc in (("out", "q_doc"), ("dq", "q_doc"), ("dk", "k_doc"), ("dv", "k_doc")):
            t = out if n == "out" else g[n].t
            assert bool((t[terms[doc] < 0] == 0).all()), n


SHAPES = [  # B, Nq, Nk, H, Hk, d
    (1, 1, 1, 1, 1, 8), (2, 1, 33, 4, 1, 32), (1, 64, 64, 2, 2, 16), (2, 65, 129, 3, 3, 40), (1, 130, 63, 6, 2, 64), (1, 257, 257, 4, 4, 32),
    (1, 100, 700, 2, 1, 128), (2, 31, 600, 8, 2, 24), (1, 1, 4097, 6, 2, 64), (1, 300, 1, 2, 1, 72), (3, 128, 128, 1, 1, 96), (1, 515, 193, 5, 5, 56),
    (1, 3, 1500, 12, 1, 128), (40, 2, 3, 2, 2, 32), (1, 1100, 70, 2, 2, 104),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(dtype, shape):
    _check(dtype, shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 65, 129, 4, 2, 32), (1, 200, 200, 2, 2, 64), (1, 70, 333, 2, 1, 128), (2, 1, 700, 6, 3, 40)])
@pytest.mark.parametrize("cap,distance,docs", [(3.0, False, None), (0.0, True, None), (0.0, False, "runs"), (0.0, False, "any"), (2.0, True, None), (0.0, True, "any"),
                                               (5.0, False, "runs"), (4.0, True, "runs")])
def test_attention_terms(dtype, shape, cap, distance, docs):
    _check(dtype, shape, cap=cap, distance=distance, docs=docs, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 88, 128])
@pytest.mark.parametrize("cap,distance,docs", [(0.0, False, None), (3.0, False, None), (0.0, True, None), (4.0, True, None), (0.0, False, "runs"), (5.0, False, "any"),
                                               (0.0, True, "runs"), (4.0, True, "any")])
def test_attention_of_many_images(dtype, d, cap, distance, docs):
    """Enough blocks of 128 rows, and of 128 keys, for the kernels that work by these."""
    _check(dtype, (130, 23, 70, 8, 4, d) if docs == "any" else (130, 37, 70, 4, 4, d), cap=cap, distance=distance, docs=docs, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,d", [(1, 32), (1, 128), (66, 32), (66, 64), (66, 128)])
@pytest.mark.parametrize("cap", [0.0, 150.0])
def test_scores_that_rise_along_the_keys(dtype, images, d, cap):
    """Scores that grow, or fall, by hundreds from the first keys to the last: what the exponentials are taken from has to follow."""
    g = np.random.default_rng(6)
    H, Nq, Nk = 8, 20, 400
    for rise in (60.0, -60.0):
        q = g.normal(size=(images, Nq, H, d)) * 0.3
        k = g.normal(size=(images, Nk, H, d)) * 0.3
        q[..., 0] = 1.0 + 0.5 * g.random((images, Nq, H))
        k[..., 0] = (np.arange(Nk) / Nk * rise)[None, :, None]
        val = {}
        dev = {}
        for n, x in (("q", q), ("k", k), ("v", g.normal(size=k.shape)), ("dout", g.normal(size=q.shape))):
            dev[n], val[n] = _stored(x, dtype)
        out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], 2.0, cap)
        got = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], 2.0, cap)
        some = slice(0, 2)
        ref = oa.attn(val["q"][some], val["k"][some], val["v"][some], 2.0, cap, dout=val["dout"][some], half=HALF[dtype], given=out[some].double().cpu().numpy())
        # what is below fp32's least normal value, 2^-126 = 1.2e-38, is 0 there: 1e3 terms of it times values of at most 1e3 are far below 1e-30
        for n, t in (("out", out), ("lse", lse), *got.items()):
            _close(t[some], ref[n][0], ref[n][1] + 1e-30, n)


def test_keys_that_all_lie_far_below_zero():
    """Scores near -1e4, and one image whose first tile is hidden from most."""
    q = torch.full((1, 70, 1, 32), 1.0, device="cuda")
    k = torch.full((1, 300, 1, 32), -312.5, device="cuda")
    v = torch.randn(1, 300, 1, 32, device="cuda")
    k[0, 200, 0, 0] += 2.0
    out, lse = aff.affmae_attn_fwd(q, k, v, 1.0)
    w = torch.ones(300, dtype=torch.float64, device="cuda")
    w[200] = float(np.exp(2.0))
    want = (w[:, None] * v[0, :, 0].double()).sum(0) / w.sum()
    # a score of 1e4 is off by at most half a step of fp32 for each of its sums: 32 * 2^-24 * 1e4 = 0.02 at worst, the same for equal keys
    assert float((out[0, :, 0].double() - want).abs().max()) < 0.04 * float(v.abs().max())
    assert float((lse[0, :, 0].double() - (-1e4 + float(w.sum().log()))).abs().max()) < 0.04


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,Nk", [(1, 70), (130, 70), (1, 1030), (66, 1030)])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("far", [-300.0, 300.0])
def test_gradients_of_scores_far_from_zero(dtype, images, Nk, d, far):
    """exp(0 - lse) of a key or query that is not there does not fit 32 bits."""
    g = np.random.default_rng(8)
    H, Nq = 4, 9
    q, k = g.normal(size=(images, Nq, H, d)) * 0.3, g.normal(size=(images, Nk, H, d)) * 0.3
    q[..., 0], k[..., 0] = 1.0, far
    dev, val = {}, {}
    for n, x in (("q", q), ("k", k), ("v", g.normal(size=k.shape)), ("dout", g.normal(size=q.shape))):
        dev[n], val[n] = _stored(x, dtype)
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], 1.0)
    got = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], 1.0)
    some = slice(0, 1)
    ref = oa.attn(val["q"][some], val["k"][some], val["v"][some], 1.0, dout=val["dout"][some], half=HALF[dtype], given=out[some].double().cpu().numpy())
    for n, t in (("out", out), ("lse", lse), *got.items()):
        assert bool(torch.isfinite(t).all()), n
        _close(t[some], *ref[n], n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_scales(dtype):
    for scale in (-0.3, 0.0, 1.5):
        _check(dtype, (1, 70, 90, 2, 2, 32), scale=scale)
        _check(dtype, (1, 70, 90, 2, 2, 32), scale=scale, cap=4.0, distance=True)
    for cap in (0.05, 1.0, 1e6, 1e30):
        _check(dtype, (1, 70, 90, 2, 2, 32), cap=cap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_images_of_many_lengths_in_one_row(dtype):
    """Runs from one token to several tiles; images that only one side has; a row of nothing but padding."""
    g = np.random.default_rng(5)
    lengths = [1, 2, 63, 64, 65, 1, 200, 7, 128, 31]
    ids = np.repeat(np.arange(len(lengths)) * 3, lengths)
    N = len(ids) + 40
    q_doc = np.full((3, N), -1, dtype=np.int32)
    k_doc = q_doc.copy()
    q_doc[0, :len(ids)] = ids
    k_doc[0, :len(ids)] = ids
    q_doc[1, 10:10 + len(ids)] = ids[::-1]   # the keys have other images in most places
    k_doc[1, :len(ids)] = np.where(ids % 2, ids, ids + 1000000)
    dev, val, _, _ = _case(dtype, 3, N, N, 2, 1, 32, seed=9)
    terms = {"q_doc": torch.from_numpy(q_doc).cuda(), "k_doc": torch.from_numpy(k_doc).cuda()}
    for n, doc in (("q", "q_doc"), ("dout", "q_doc"), ("k", "k_doc"), ("v", "k_doc")):
        dev[n][terms[doc] < 0] = float("nan")
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], 0.2, **terms)
    got = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], 0.2, **terms)
    ref = oa.attn(val["q"], val["k"], val["v"], float(np.float32(0.2)), q_doc=q_doc, k_doc=k_doc, dout=val["dout"], half=HALF[dtype], given=out.double().cpu().numpy())
    for n, t in (("out", out), ("lse", lse), *got.items()):
        _close(t, *ref[n], n)
    assert bool((out[2] == 0).all()) and bool((lse[2] == -np.inf).all())


def test_results_do_not_change_from_run_to_run():
    for shape, docs in (((2, 300, 500, 4, 2, 64), "runs"), ((1, 1, 9000, 4, 1, 32), None), ((1, 2500, 40, 2, 2, 128), None)):
        dev, _, terms, _ = _case("bf16", *shape, cap=10.0, distance=True, docs=docs, poison=False)
        runs = []
        for _ in range(3):
            out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], 0.1, 10.0, **terms)
            g = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], 0.1, 10.0, **terms)
            runs.append([out, lse, *g.values()])
        for other in runs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_gradients_against_differences():
    """fp32: a step along a random direction of every input, against what the forward kernel itself returns.

    The loss <dout, out> is off by at most e = 5e-6 of the sum |dout| |out| (the forward's bound at these sizes), twice in a difference over 2
    steps; the third derivative adds step^2 / 6 times at most about 30 of the first."""
    dev, _, terms, _ = _case("f32", 1, 60, 90, 2, 1, 32, cap=3.0, distance=True, docs="any", poison=False)
    scale, step = 0.25, 2e-2
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], scale, 3.0, **terms)
    g = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], scale, 3.0, **terms)
    gen = torch.Generator(device="cuda").manual_seed(1)
    size = float((dev["dout"].double().abs() * out.double().abs()).sum())
    for name in ("q", "k", "v", "slope"):
        x = terms[name] if name == "slope" else dev[name]
        way = torch.randn(x.shape, generator=gen, device="cuda")
        way = way / way.norm() * (0.05 if name == "slope" else 1.0)
        values = []
        for sign in (1, -1):
            moved = {"q": dev["q"], "k": dev["k"], "v": dev["v"], "slope": terms["slope"]}
            moved[name] = x + sign * step * way
            o, _ = aff.affmae_attn_fwd(moved["q"], moved["k"], moved["v"], scale, 3.0, **{**terms, "slope": moved["slope"]})
            values.append(float((o.double() * dev["dout"].double()).sum()))
        real = (x + step * way).double() - (x - step * way).double()  # (as rounded)
        want = float((g["d" + name].double() * real).sum())
        seen = values[0] - values[1]
        assert abs(seen - want) <= 2 * 5e-6 * size * 0.1 + step ** 2 / 6 * 30 * abs(want) + 1e-5 * size * step, (name, seen, want)


def test_keys_beyond_32_bits():
    """k and v of more than 2^32 bytes each: the last keys are the ones that count."""
    Nk, H, d = (1 << 20) + 5, 17, 128
    k = torch.zeros(1, Nk, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q = torch.zeros(1, 2, H, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    k[0, -3:, :, 0] = 20.0
    v[0, -3:, :, :] = torch.arange(1, 4, device="cuda", dtype=torch.bfloat16)[:, None, None] * 8
    out, lse = aff.affmae_attn_fwd(q, k, v, 1.0)
    e = np.exp(20.0)
    want = 16.0 * 3 * e / (3 * e + Nk - 3)
    assert np.allclose(out.float().cpu().numpy(), want, rtol=2 ** -7) and np.allclose(lse.cpu().numpy(), np.log(3 * e + Nk - 3), rtol=1e-6)
    dout = torch.ones_like(q)
    g = aff.affmae_attn_bwd(q, k, v, out, lse, dout, 1.0)
    p = e / (3 * e + Nk - 3)
    assert np.allclose(g["dv"][0, -3:].float().cpu().numpy(), 2 * p, rtol=2 ** -6)
    assert float(g["dv"][0, :-3].float().abs().max()) <= 2 * 1.1 / (3 * e)
    del k, v, g
    torch.cuda.empty_cache()


def test_on_another_stream_and_in_a_graph():
    """A whole branch, linear -> rotary -> attention, forward and backward, on a stream of its own; then captured and replayed, with eager
    calls in between, new inputs and two graphs over one workspace."""
    B, N, H, Hk, d = 2, 150, 4, 2, 32
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(B, N, H * d, generator=gen, device="cuda").to(torch.bfloat16)
    w = [(torch.randn(n, H * d, generator=gen, device="cuda") * (H * d) ** -0.5).to(torch.bfloat16) for n in (H * d, Hk * d, Hk * d)]
    coords = torch.rand(B, N, 2, generator=gen, device="cuda") * 512
    freq = torch.rand(d // 2, 2, generator=gen, device="cuda")
    slope = torch.tensor([0.01, 0.02, 0.0, 0.05], device="cuda")
    docs = torch.arange(N, device="cuda", dtype=torch.int32)[None].expand(B, N).div(40, rounding_mode="floor").to(torch.int32).contiguous()
    docs[:, -9:] = -1
    dout = torch.randn(B, N, H, d, generator=gen, device="cuda").to(torch.bfloat16)
    terms = dict(q_xy=coords, k_xy=coords, slope=slope, q_doc=docs, k_doc=docs)

    def branch():
        q, k, v = (aff.affmae_linear_fwd(x, m)[0].view(B, N, -1, d) for m in w)
        qr, kr = aff.affmae_rotary_fwd(q, coords, freq, k=k)
        out, lse = aff.affmae_attn_fwd(qr, kr, v, d ** -0.5, 20.0, **terms)
        g = aff.affmae_attn_bwd(qr, kr, v, out, lse, dout, d ** -0.5, 20.0, **terms)
        r = aff.affmae_rotary_bwd(g["dq"], coords, freq, dk_out=g["dk"], q_out=qr, k_out=kr, want_dcoords=True)
        dx = aff.affmae_linear_bwd(x, w[0], r["dq"].view(B, N, -1))
        return [out, lse, *g.values(), *r.values(), *dx.values()]

    eager = [t.clone() for t in branch()]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = branch()
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = branch()
    for turn in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, captured)), turn
        if turn == 1:
            x.mul_(0.5)
        eager = [t.clone() for t in branch()]
        torch.cuda.synchronize()


def test_two_graphs_over_one_workspace():
    dev, _, terms, _ = _case("bf16", 1, 64, 3000, 2, 1, 64, distance=True, docs="runs", poison=False)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    outs = []
    for scale in (0.1, 0.3):
        out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], scale, **terms)
        outs.append((scale, out, lse, aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], scale, **terms)))
    graphs = []
    for scale, *_ in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, l = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], scale, workspace=ws, **terms)
            g = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], o, l, dev["dout"], scale, workspace=ws, **terms)
        graphs.append((graph, o, l, g))
    for _ in range(3):
        for (graph, o, l, g), (_, out, lse, want) in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, out) and torch.equal(l, lse) and all(torch.equal(g[n], want[n]) for n in want)
            ws.fill_(255)


# ------------------------------------------------------------------------------------------------------ rotary positions

ROTARY = [  # B, N, H, Hk, d, axes
    (1, 1, 1, 0, 2, 1), (2, 5, 3, 1, 6, 2), (1, 257, 2, 2, 32, 2), (3, 100, 6, 0, 64, 3), (2, 33, 4, 2, 24, 2), (1, 70, 12, 4, 128, 3), (1, 300, 1, 1, 34, 1),
    (2, 9, 5, 3, 512, 2), (1, 1000, 2, 1, 20, 2), (1, 40, 7, 7, 12, 3),
]


def _rotary_case(dtype, B, N, H, Hk, d, axes, far):
    g = np.random.default_rng(N * 31 + d)
    dev, val = {}, {}
    for n, shape in (("q", (B, N, H, d)), ("k", (B, N, Hk, d)), ("dq", (B, N, H, d)), ("dk", (B, N, Hk, d))):
        dev[n], val[n] = _stored(g.normal(size=shape), dtype)
    dev["coords"], val["coords"] = _stored(g.uniform(0, 1000, (B, N, axes)) + far, "f32")
    dev["freq"], val["freq"] = _stored(g.uniform(-0.5, 0.5, (d // 2, axes)) * (g.random((d // 2, axes)) < 0.6), "f32")
    return dev, val


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("far", [0.0, -3.0e6])
@pytest.mark.parametrize("shape", ROTARY)
def test_rotary(dtype, layout, far, shape):
    """sin and cos are off by 2^-22 and |angle| 2^-51 (its own sum, and the one that it is compared with); a value is two products and a sum."""
    B, N, H, Hk, d, axes = shape
    dev, val = _rotary_case(dtype, *shape, far)
    turn = np.abs(val["coords"]) @ np.abs(val["freq"]).T
    angle = (2.0 ** -22 + 2.0 ** -51 * turn.max() + 4 * U)

    def bound(x, back):
        y = oa.rotary(x, val["coords"], val["freq"], layout, back)
        a, b = oa._pairs(d, layout)
        t = np.zeros_like(x)
        t[..., a] = t[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * angle
        return y, t + HALF[dtype] * (np.abs(y) + t)

    names = ("q", "k") if Hk else ("q",)
    to = {n: Guarded(dev[n].shape, TYPES[dtype]) for n in names}
    aff.affmae_rotary_fwd(dev["q"], dev["coords"], dev["freq"], k=dev["k"] if Hk else None, layout=layout, q_out=to["q"].t, k_out=to["k"].t if Hk else None)
    for n in names:
        _close(to[n].t, *bound(val[n], False), n)
        to[n].check()
    grads = {"d" + n: Guarded(dev[n].shape, TYPES[dtype]) for n in names}
    grads["dcoords"] = Guarded((B, N, axes), torch.float32)
    out = {n + "_out": to[n].t for n in names}
    aff.affmae_rotary_bwd(dev["dq"], dev["coords"], dev["freq"], dk_out=dev["dk"] if Hk else None, layout=layout, want_dcoords=True,
                          grads={n: x.t for n, x in grads.items()}, **out)
    spin, size = 0.0, 0.0
    for n in names:
        _close(grads["d" + n].t, *bound(val["d" + n], True), "d" + n)
        s, z = oa.rotary_spin(to[n].t.double().cpu().numpy(), val["d" + n], layout)
        spin, size = spin + s, size + z
    _close(grads["dcoords"].t, spin @ val["freq"], 2 * U * (H + Hk + d // 2 + 8) * (size @ np.abs(val["freq"])), "dcoords")
    for x in grads.values():
        x.check()
    # the same without the places' gradient, and in place
    g = aff.affmae_rotary_bwd(dev["dq"], dev["coords"], dev["freq"], dk_out=dev["dk"] if Hk else None, layout=layout)
    assert all(torch.equal(g["d" + n], grads["d" + n].t) for n in names)
    q, k = dev["q"].clone(), dev["k"].clone()
    aff.affmae_rotary_fwd(q, dev["coords"], dev["freq"], k=k if Hk else None, layout=layout, q_out=q, k_out=k if Hk else None)
    assert torch.equal(q, to["q"].t) and (not Hk or torch.equal(k, to["k"].t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [1, 3])
def test_rotary_off_its_alignment(dtype, shift):
    dev, _ = _rotary_case(dtype, 2, 50, 3, 1, 32, 2, 0.0)
    q, _ = aff.affmae_rotary_fwd(dev["q"], dev["coords"], dev["freq"])
    buf = torch.zeros(dev["q"].numel() + 16, dtype=TYPES[dtype], device="cuda")
    moved = buf[shift:shift + dev["q"].numel()].view(dev["q"].shape)
    moved.copy_(dev["q"])
    aff.affmae_rotary_fwd(moved, dev["coords"], dev["freq"], q_out=moved)
    assert torch.equal(moved, q) and bool((buf[:shift] == 0).all()) and bool((buf[shift + q.numel():] == 0).all())


def test_rotary_of_many_tokens():
    """More tokens than the launch's blocks hold at once, and identity where freq is 0."""
    N = 9_000_001
    q = torch.randn(1, N, 1, 8, device="cuda")
    coords = torch.rand(1, N, 1, device="cuda")
    freq = torch.tensor([[0.0], [3.0], [0.0], [0.5]], device="cuda")
    out, _ = aff.affmae_rotary_fwd(q, coords, freq)
    assert torch.equal(out[..., 0:2], q[..., 0:2]) and torch.equal(out[..., 4:6], q[..., 4:6])
    t = (coords.double() * 3.0)[..., None]
    want = q[..., 2:3].double() * t.cos() - q[..., 3:4].double() * t.sin()
    assert float((out[..., 2:3].double() - want).abs().max()) < 6 * 2.0 ** -22
