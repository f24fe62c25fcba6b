"""CPU-side checks of the C ABI and binding of attention between all tokens and of rotary positions: every bad argument is refused on the
host before anything is enqueued."""
import pytest
import torch

import paper_2602_16249_amd as aff
from paper_2602_16249_amd import binding

P = 4096          # never dereferenced: validation fails first
NAN, INF = float("nan"), float("inf")
FAR = 2 ** 32     # its low 32 bits are 0


def test_rotary_refuses():
    lib = aff.load_library()

    def fwd(q=P, k=P, coords=P, freq=P, B=2, N=5, H=4, Hk=2, d=8, axes=2, layout=0, dtype=1, qo=P, ko=P):
        return lib.affmae_rotary_fwd(q, k, coords, freq, B, N, H, Hk, d, axes, layout, dtype, qo, ko, None)

    for name in ("q", "k", "coords", "freq", "qo", "ko"):
        assert fwd(**{name: None}) == -1, name
        assert fwd(**{name: P + 1}) == -2, name
    assert fwd(Hk=0) == -1                                         # keys without heads
    assert fwd(B=0) == -2 and fwd(N=0) == -2 and fwd(H=0) == -2 and fwd(Hk=-1) == -2 and fwd(axes=0) == -2
    assert fwd(d=7) == -2 and fwd(d=0) == -2 and fwd(layout=2) == -2 and fwd(layout=-1) == -2
    assert fwd(dtype=2) == -3
    assert fwd(d=514) == -5 and fwd(axes=4) == -5 and fwd(H=4097) == -5 and fwd(B=1 << 16, N=1 << 15) == -5
    assert fwd(B=1 << 15, N=1 << 15, H=30, Hk=2, d=512) == -5

    def bwd(dqo=P, dko=P, qo=P, ko=P, coords=P, freq=P, H=4, Hk=2, d=8, dtype=0, dq=P, dk=P, dc=P):
        return lib.affmae_rotary_bwd(dqo, dko, qo, ko, coords, freq, 2, 5, H, Hk, d, 2, 0, dtype, dq, dk, dc, None)

    for name in ("dqo", "dko", "qo", "ko", "coords", "freq", "dq", "dk"):
        assert bwd(**{name: None}) == -1, name
    for name in ("dqo", "dko", "qo", "ko", "coords", "freq", "dq", "dk", "dc"):
        assert bwd(**{name: P + 2}) == -2, name
    assert bwd(Hk=0) == -1 and bwd(d=3) == -2 and bwd(dtype=-1) == -3 and bwd(d=1024) == -5


def test_attention_refuses():
    lib = aff.load_library()

    def fwd(q=P, k=P, v=P, qx=P, kx=P, sl=P, qd=P, kd=P, B=2, Nq=100, Nk=70, H=4, Hk=2, d=32, scale=1.0, cap=0.0, dtype=1, out=P, lse=P, ws=P, size=1 << 30):
        return lib.affmae_attn_fwd(q, k, v, qx, kx, sl, qd, kd, B, Nq, Nk, H, Hk, d, scale, cap, dtype, out, lse, ws, size, None)

    for name in ("q", "k", "v", "qx", "kx", "sl", "qd", "kd", "out", "lse"):
        assert fwd(**{name: None}) == -1, name
    for name in ("q", "k", "v", "out"):
        assert fwd(**{name: P + 8}) == -2, name
    for name in ("qx", "kx"):
        assert fwd(**{name: P + 4}) == -2, name
    for name in ("sl", "qd", "kd", "lse"):
        assert fwd(**{name: P + 2}) == -2, name
    for name in ("B", "Nq", "Nk", "H", "Hk", "d"):
        assert fwd(**{name: 0}) == -2, name
    assert fwd(Hk=3) == -2 and fwd(Hk=8) == -2
    assert fwd(scale=NAN) == -2 and fwd(scale=INF) == -2 and fwd(cap=-1.0) == -2 and fwd(cap=NAN) == -2 and fwd(cap=INF) == -2 and fwd(cap=1e-35) == -2 and fwd(scale=1e20, cap=1e-20) == -2
    assert fwd(dtype=2) == -3
    assert fwd(d=20) == -5 and fwd(d=136) == -5 and fwd(H=4098) == -5 and fwd(Nk=(1 << 24) + 1) == -5 and fwd(Nq=(1 << 24) + 1) == -5
    assert fwd(B=1 << 24) == -5 and fwd(Nq=1 << 24, H=256, Hk=2) == -5
    need = lib.affmae_attn_fwd_workspace_bytes(2, 100, 70, 4, 2, 32, 1, 1)
    assert need > 0 and lib.affmae_attn_fwd_workspace_bytes(2, 100, 0, 4, 2, 32, 1, 1) == 0
    assert fwd(ws=None) == -4 and fwd(size=need - 1) == -4 and fwd(ws=P + 128) == -4

    def bwd(q=P, k=P, v=P, qx=P, kx=P, sl=P, qd=P, kd=P, out=P, lse=P, dout=P, Nq=100, H=4, d=32, cap=0.0, dtype=1, dq=P, dk=P, dv=P, ds=P, ws=P, size=1 << 30):
        return lib.affmae_attn_bwd(q, k, v, qx, kx, sl, qd, kd, out, lse, dout, 2, Nq, 70, H, 2, d, 1.0, cap, dtype, dq, dk, dv, ds, ws, size, None)

    for name in ("q", "k", "v", "qx", "kx", "sl", "qd", "kd", "out", "lse", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == -1, name
    assert bwd(qx=None, kx=None, sl=None) == -1                    # a gradient of what is not there
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: P + 4}) == -2, name
    assert bwd(ds=P + 1) == -2 and bwd(lse=P + 1) == -2 and bwd(cap=-0.5) == -2 and bwd(H=5) == -2 and bwd(Nq=0) == -2
    assert bwd(dtype=7) == -3 and bwd(d=12) == -5
    need = lib.affmae_attn_bwd_workspace_bytes(2, 100, 70, 4, 2, 32, 1, 1, 1)
    assert need >= 2 * 100 * 4 * 4 and bwd(ws=None) == -4 and bwd(size=need - 1) == -4 and bwd(ws=P + 64) == -4
    assert lib.affmae_attn_bwd_workspace_bytes(2, 100, 70, 4, 3, 32, 1, 1, 1) == 0


def test_binding_refuses_host_tensors():
    x, xy = torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 2)
    for call in (lambda: aff.affmae_attn_fwd(x, x, x, 1.0), lambda: aff.affmae_attn_bwd(x, x, x, x, x, x, 1.0), lambda: aff.affmae_attn_fwd(x.half(), x.half(), x.half(), 1.0),
                 lambda: aff.affmae_rotary_fwd(x, xy, torch.zeros(4, 2)), lambda: aff.affmae_rotary_bwd(x, xy, torch.zeros(4, 2))):
        with pytest.raises(ValueError):
            call()


class NotToBeCalled:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(binding, "load_library", lambda: NotToBeCalled())
    monkeypatch.setattr(binding, "status_string", lambda status: "")  # (error texts come from the library)
    monkeypatch.setattr(binding, "_current", lambda t: 0)
    monkeypatch.setattr(binding, "_on", lambda index, t, name, dtype, shape=None: 4096)


def _meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("B,N,H,d", [(FAR + 1, 1, 1, 8), (1, FAR + 1, 1, 8), (1, 1, FAR + 1, 8), (1, 1, 1, FAR + 8)])
def test_sizes_beyond_an_int(no_library, B, N, H, d):
    x, xy, one = _meta(B, N, H, d), _meta(B, N, 2, dtype=torch.float32), _meta(1, 1, 1, 8)
    calls = [lambda: aff.affmae_attn_fwd(x, one, one, 1.0), lambda: aff.affmae_attn_bwd(x, one, one, x, x, x, 1.0),
             lambda: aff.affmae_rotary_fwd(x, xy, xy), lambda: aff.affmae_rotary_bwd(x, xy, xy)]
    if B == 1 and d == 8:
        calls.append(lambda: aff.affmae_attn_fwd(one, x, x, 1.0))
    for call in calls:
        with pytest.raises(aff.AffmaeError) as e:
            call()
        assert e.value.status == -5


def test_binding_refuses_halves_of_terms(no_library):
    x, xy, s, ids = _meta(1, 4, 2, 8), _meta(1, 4, 2, dtype=torch.float32), _meta(2, dtype=torch.float32), _meta(1, 4, dtype=torch.int32)
    for terms in (dict(slope=s), dict(q_xy=xy, k_xy=xy), dict(slope=s, q_xy=xy), dict(q_doc=ids), dict(k_doc=ids)):
        with pytest.raises(ValueError):
            aff.affmae_attn_fwd(x, x, x, 1.0, **terms)
        with pytest.raises(ValueError):
            aff.affmae_attn_bwd(x, x, x, x, x, x, 1.0, **terms)
    with pytest.raises(ValueError):
        aff.affmae_rotary_fwd(x, xy, xy, layout="thirds")
    with pytest.raises(ValueError):
        aff.affmae_rotary_fwd(x, xy, xy, k_out=x)
    with pytest.raises(ValueError):
        aff.affmae_rotary_bwd(x, xy, xy, want_dcoords=True)
    with pytest.raises(ValueError):
        aff.affmae_rotary_bwd(x, xy, xy, dk_out=x, q_out=x, want_dcoords=True)


def test_rotary_layouts_of_header_and_binding():
    import os
    import re
    text = open(os.path.join(os.path.dirname(aff.library_path()), "..", "include", "affmae.h")).read()
    assert {n.lower(): int(v) for n, v in re.findall(r"AFFMAE_ROTARY_([A-Z]+) = (\d)", text)} == binding._ROTARY_LAYOUTS


def test_binding_refuses_gradients_that_a_call_does_not_write(no_library):
    """A buffer that stays as it was would come back as if it held a gradient."""
    x, xy, s, freq = _meta(1, 4, 2, 8), _meta(1, 4, 2, dtype=torch.float32), _meta(2, dtype=torch.float32), _meta(4, 2, dtype=torch.float32)
    where = dict(q_xy=xy, k_xy=xy, slope=s)
    for grads, more in ((dict(dslope=s), {}), (dict(dslope=s), dict(want_dslope=False, **where)), (dict(dq=x, dkey=x), {}), (dict(dbias=x), where)):
        with pytest.raises(ValueError, match="not written"):
            aff.affmae_attn_bwd(x, x, x, x, x, x, 1.0, grads=grads, **more)
    for grads, more in ((dict(dcoords=xy), {}), (dict(dq=x, dk=x), {}), (dict(dcoords=xy), dict(dk_out=x)), (dict(dfreq=freq), dict(q_out=x, want_dcoords=True))):
        with pytest.raises(ValueError, match="not written"):
            aff.affmae_rotary_bwd(x, xy, freq, grads=grads, **more)


@pytest.mark.parametrize("scale,cap", [(3e38, 0.0), (-2.5e38, 0.0), (3e38, 3e38), (1.0, 2.5e38), (1.0, 3.4e38), (1.0, 2e38)])
def test_attention_refuses_scales_and_caps_beyond_its_own_numbers(scale, cap):
    """scale log2 e and 2 cap log2 e have to be finite: the scores are in units of log 2."""
    lib = aff.load_library()
    assert lib.affmae_attn_fwd(P, P, P, None, None, None, None, None, 2, 100, 70, 4, 2, 32, scale, cap, 1, P, P, P, 1 << 30, None) == -2
    assert lib.affmae_attn_bwd(P, P, P, None, None, None, None, None, P, P, P, 2, 100, 70, 4, 2, 32, scale, cap, 1, P, P, P, None, P, 1 << 30, None) == -2
