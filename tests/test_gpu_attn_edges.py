"""GPU tests of the attention where its kernels differ from the usual path: images whose keys begin late, long rows of wide heads, tensors beyond
2^32 bytes with all their gradients.  Bounds as in tests/test_gpu_attn.py."""
import numpy as np
import pytest
import torch

import paper_2602_16249_amd as aff
from oracle import attn as oa
from test_gpu_attn import HALF, _case, _check, _close, _stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images", [1, 130])
@pytest.mark.parametrize("cap", [0.0, 3.0e4])
def test_keys_hidden_from_most_queries_come_first(dtype, images, cap):
    """Scores near -1e4; the first two tiles belong to the image of three queries, and a row of another image sees its first key in the third."""
    g = np.random.default_rng(12)
    Nq, Nk, H, d = 70, 300, 4, 32
    q_doc, k_doc = np.full((images, Nq), 1, dtype=np.int32), np.full((images, Nk), 1, dtype=np.int32)
    q_doc[:, [0, 33, 69]] = 0
    q_doc[:, 5] = 2  # (no key)
    k_doc[:, :130] = 0
    dev, val = {}, {}
    for n, x in (("q", np.ones((images, Nq, H, d))), ("k", -312.5 + 0.1 * g.normal(size=(images, Nk, H, d))), ("v", g.normal(size=(images, Nk, H, d))),
                 ("dout", g.normal(size=(images, Nq, H, d)))):
        dev[n], val[n] = _stored(x, dtype)
    terms = {n: torch.from_numpy(x).cuda() for n, x in (("q_doc", q_doc), ("k_doc", k_doc))}
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], 1.0, cap, **terms)
    got = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], 1.0, cap, **terms)
    some = slice(images - 1, images)
    ref = oa.attn(val["q"][some], val["k"][some], val["v"][some], 1.0, cap, dout=val["dout"][some], half=HALF[dtype], given=out[some].double().cpu().numpy(),
                  q_doc=q_doc[some], k_doc=k_doc[some])
    for n, t in (("out", out), ("lse", lse), *got.items()):
        _close(t[some], *ref[n], n)
    assert bool((out[:, 5] == 0).all()) and bool((lse[:, 5] == -np.inf).all()) and bool((got["dq"][:, 5] == 0).all())


@pytest.mark.parametrize("d", [72, 104, 128])
@pytest.mark.parametrize("shape", [(1, 70, 1025, 2, 1), (1, 5, 2999, 4, 2), (66, 20, 1030, 4, 4)])
def test_capped_long_rows_of_wide_heads(d, shape):
    if shape[0] == 1:
        _check("bf16", (*shape, d), cap=3.0, seed=3)
    else:  # (the plain implementation takes its time with many images: the first ones)
        B, Nq, Nk, H, Hk = shape
        g = np.random.default_rng(d)
        dev, val = {}, {}
        for n, x in (("q", (B, Nq, H, d)), ("k", (B, Nk, Hk, d)), ("v", (B, Nk, Hk, d)), ("dout", (B, Nq, H, d))):
            dev[n], val[n] = _stored(g.normal(size=x), "bf16")
        scale = float(np.float32(d ** -0.5))
        out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], scale, 3.0)
        got = aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], scale, 3.0)
        ref = oa.attn(val["q"][:1], val["k"][:1], val["v"][:1], scale, 3.0, dout=val["dout"][:1], half=HALF["bf16"], given=out[:1].double().cpu().numpy(),
                      puts_right=True)
        for n, t in (("out", out), ("lse", lse), *got.items()):
            _close(t[:1], *ref[n], n)


def test_gradients_of_keys_beyond_32_bits():
    """k and v of more than 2^32 bytes each.  Three keys at the end share all but (Nk - 3) / (3 e^20) = 0.0007 of the weight, each with a channel
    of its own that no query has."""
    Nk, H, d = (1 << 20) + 5, 17, 128
    k = torch.zeros(1, Nk, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q = torch.zeros(1, 2, H, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    k[0, -3:, :, 0] = 20.0
    values = np.array([8.0, 16.0, 32.0])
    for i in range(3):
        k[0, Nk - 3 + i, :, 1 + i] = 8.0
        v[0, Nk - 3 + i] = values[i]
    dout = torch.ones_like(q)
    out, lse = aff.affmae_attn_fwd(q, k, v, 1.0)
    got = aff.affmae_attn_bwd(q, k, v, out, lse, dout, 1.0)
    e = np.exp(20.0)
    p, least = e / (3 * e + Nk - 3), 1 / (3 * e + Nk - 3)
    D = d * p * values.sum()
    dS = p * (d * values - D)
    # p and dS are rounded, and so is what comes out; sums over a million keys of least D each may lose all of these: 0.0007 D
    lost = p * (Nk - 3) * least * D
    dq = got["dq"][0].double().cpu().numpy()
    assert np.allclose(got["dv"][0, -3:].double().cpu().numpy(), 2 * p, rtol=2 ** -7 + 1e-4, atol=0)
    assert (np.abs(dq[:, :, 1:4] - 8 * dS) <= 8 * (2 ** -7 * np.abs(dS) + 2 ** -8 * p * D + lost)).all()
    assert (dq[:, :, 4:] == 0).all()
    dk = got["dk"][0]
    assert (np.abs(dk[-3:, :, 0].double().cpu().numpy() - 2 * dS[:, None]) <= 2 * (2 ** -7 * np.abs(dS)[:, None] + lost)).all()
    assert bool((dk[:, :, 1:] == 0).all())
    others = dk[:-3, :, 0].float()
    assert float((others + 2 * least * D).abs().max()) <= 2 * least * D * (2 ** -7 + 0.002)
    del k, v, got, dk, others
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1, 4097, 6, 2, 64), (2, 65, 129, 3, 3, 40), (1, 9, 2999, 4, 2, 128), (1, 2500, 40, 2, 2, 128), (66, 20, 150, 4, 4, 32)])
@pytest.mark.parametrize("docs", [None, "any"])
def test_workspaces_of_just_the_size_asked_for(dtype, shape, docs):
    """Nothing behind the workspace is written, with the gradient of the slopes and without it, and the other gradients are the same."""
    dev, _, terms, _ = _case(dtype, *shape, cap=6.0, distance=True, docs=docs, poison=False)
    lib = aff.load_library()
    code = {"f32": 0, "bf16": 1}[dtype]

    def guarded(need):
        buf = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
        return buf, buf[:need]

    def whole(buf, need):
        return bool((buf[need:] == 171).all())

    need = lib.affmae_attn_fwd_workspace_bytes(*shape, code, docs is not None)
    buf, ws = guarded(need)
    out, lse = aff.affmae_attn_fwd(dev["q"], dev["k"], dev["v"], 0.2, 6.0, workspace=ws, **terms)
    assert whole(buf, need)
    results = []
    for want in (True, False):
        need = lib.affmae_attn_bwd_workspace_bytes(*shape, code, docs is not None, want)
        buf, ws = guarded(need)
        results.append(aff.affmae_attn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], 0.2, 6.0, want_dslope=want, workspace=ws, **terms))
        assert whole(buf, need)
    assert sorted(results[1]) == ["dk", "dq", "dv"] and all(torch.equal(results[0][n], results[1][n]) for n in results[1])
