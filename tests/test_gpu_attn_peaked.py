"""GPU parity of the attention's gradients where few keys share a row's weight, by the bounds of calls that put D = <dout, out> right (oracle/attn.py;
tests/test_oracle_attn.py shows on the CPU that these bounds tell a D from the bf16 output, and one put right with the wrong sign, apart)."""
import numpy as np
import pytest
import torch

import paper_2602_16249_amd as aff
from oracle import attn as oa
from test_gpu_attn import HALF, Guarded, _close, _stored

pytestmark = pytest.mark.gpu


def _check(dtype, B, Nq, Nk, H, Hk, d, cap=0.0, distance=False, docs=False, images=None):
    """Queries near the sum of two keys.  `images`: how many of B are compared value by value (all)."""
    g = np.random.default_rng(B + 31 * Nq + Nk + d)
    G = H // Hk
    q, k = np.empty((B, Nq, H, d)), g.normal(size=(B, Nk, Hk, d))
    dev, val, terms, tval = {}, {}, {}, {}
    if docs:  # images of uneven length side by side, the last places padding
        ends = [np.sort(g.integers(1, n, 4)) for n in (Nq, Nk)]
        for n, x, e in (("q_doc", Nq, ends[0]), ("k_doc", Nk, ends[1])):
            ids = np.searchsorted(e, np.arange(x), side="right").astype(np.int32)
            ids[x - x // 16:] = -1
            tval[n] = np.broadcast_to(ids, (B, x)).copy()
    for b in range(B):
        for h in range(H):
            first, second = (g.integers(0, Nk, Nq) for _ in range(2))
            if docs:  # of the query's image, where that has keys
                for i in range(Nq):
                    own = np.flatnonzero(tval["k_doc"][b] == tval["q_doc"][b, i])
                    if len(own):
                        first[i], second[i] = g.choice(own, 2)
            kh = k[b, :, h // G]
            q[b, :, h] = kh[first] + kh[second] * g.uniform(0.6, 1.0, (Nq, 1)) + 0.1 * g.normal(size=(Nq, d))
    for n, x in (("q", q), ("k", k), ("v", g.normal(size=k.shape)), ("dout", g.normal(size=q.shape))):
        dev[n], val[n] = _stored(x, dtype)
    if distance:
        for n, x in (("q_xy", g.uniform(0, 10, (B, Nq, 2))), ("k_xy", g.uniform(0, 10, (B, Nk, 2))), ("slope", g.uniform(0.01, 0.08, H))):
            terms[n], tval[n] = _stored(x, "f32")
    if docs:
        terms.update({n: torch.from_numpy(tval[n]).cuda() for n in ("q_doc", "k_doc")})
    scale = float(np.float32(d ** -0.5))
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], scale, cap, **terms)
    to = {n: Guarded(dev[n[1:]].shape, dev["q"].dtype) for n in ("dq", "dk", "dv")}
    got = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], scale, cap, grads={n: x.t for n, x in to.items()}, **terms)
    some = slice(0, B if images is None else images)
    assert images is None or not distance  # (dslope is a sum over all images)
    part = {n: x if n == "slope" else x[some] for n, x in tval.items()}
    ref = oa.attn(val["q"][some], val["k"][some], val["v"][some], scale, cap, dout=val["dout"][some], half=HALF[dtype],
                  given=out[some].double().cpu().numpy(), puts_right=dtype == "bf16", **part)
    _close(out[some], *ref["out"], "out")
    _close(lse[some], *ref["lse"], "lse")
    for n, t in got.items():
        _close(t if n == "dslope" else t[some], *ref[n], n)
    for x in to.values():
        x.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 40, 64])
@pytest.mark.parametrize("Nk", [2, 1023, 1024, 4097])
def test_two_keys_share_the_weight(dtype, d, Nk):
    _check(dtype, 1, 70, Nk, 4, 2, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Nk", [(50, 301), (9, 900), (200, 77)])
@pytest.mark.parametrize("cap,distance,docs", [(30.0, False, False), (0.0, True, False), (0.0, False, True), (25.0, True, True)])
def test_two_keys_share_the_weight_with_terms(dtype, d, Nq, Nk, cap, distance, docs):
    """Nq of 9: the keys are split over workgroups, and what D lacks comes from several sums."""
    _check(dtype, 2, Nq, Nk, 4, 2, d, cap, distance, docs)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("cap,docs", [(0.0, False), (30.0, False), (0.0, True)])
def test_two_keys_share_the_weight_in_many_images(d, cap, docs):
    """Enough blocks of 128 rows, and of 128 keys, for the kernels that work by these."""
    _check("bf16", 130, 23, 150, 4, 4, d, cap, False, docs, images=2)


@pytest.mark.parametrize("d", [72, 104, 128])
@pytest.mark.parametrize("Nk", [2, 1023, 1024, 4097])
def test_two_keys_share_the_weight_in_wide_heads(d, Nk):
    """D is put right whatever the row's length."""
    _check("bf16", 1, 70, Nk, 4, 2, d)


@pytest.mark.parametrize("d", [72, 128])
@pytest.mark.parametrize("Nq,Nk", [(70, 1025), (9, 2999)])
@pytest.mark.parametrize("cap,distance,docs", [(30.0, False, False), (0.0, True, False), (0.0, False, True), (25.0, True, True)])
def test_long_rows_of_wide_heads_with_terms(d, Nq, Nk, cap, distance, docs):
    _check("bf16", 2, Nq, Nk, 4, 2, d, cap, distance, docs)


@pytest.mark.parametrize("d", [72, 128])
@pytest.mark.parametrize("cap,docs", [(0.0, False), (30.0, False), (0.0, True)])
def test_long_rows_of_wide_heads_in_many_images(d, cap, docs):
    _check("bf16", 66, 20, 1030, 4, 4, d, cap, False, docs, images=1)
