"""CPU-side checks of the dense operators' C ABI: every bad argument is refused on the host before anything is enqueued."""
import ctypes

import pytest
import torch

import paper_2602_16249_amd as aff

P = 4096          # never dereferenced: validation fails first
NAN = float("nan")


def test_linear_forward_refuses():
    lib = aff.load_library()

    def fwd(x=P, w=P, bias=None, res=None, rows=10, Cin=8, Cout=8, act=0, p=0.0, rng=None, dtype=1, out=P, pre=None):
        return lib.affmae_linear_fwd(x, w, bias, res, rows, Cin, Cout, act, p, rng, dtype, out, pre, None)

    assert fwd(x=None) == -1 and fwd(w=None) == -1 and fwd(out=None) == -1
    assert fwd(p=0.5) == -1                                       # dropout without the generator's state
    assert fwd(rows=0) == -2 and fwd(Cin=0) == -2 and fwd(Cout=-1) == -2
    assert fwd(act=4) == -2 and fwd(act=-1) == -2
    assert fwd(p=1.0, rng=P) == -2 and fwd(p=-0.1, rng=P) == -2 and fwd(p=NAN, rng=P) == -2
    assert fwd(rng=P + 4, p=0.5) == -2
    for name in ("x", "w", "bias", "res", "out", "pre"):
        assert fwd(**{name: P + 1}) == -2, name
        assert fwd(dtype=0, **{name: P + 2}) == -2, name
    assert fwd(dtype=2) == -3
    assert fwd(Cin=(1 << 20) + 1) == -5 and fwd(Cout=(1 << 20) + 1) == -5 and fwd(rows=(1 << 29) + 1) == -5
    assert fwd(rows=1 << 29, Cin=65) == -5 and fwd(rows=1 << 29, Cout=65) == -5
    assert fwd(Cin=1 << 18, Cout=(1 << 17) + 1) == -5


def test_linear_backward_refuses():
    lib = aff.load_library()

    def bwd(x=P, w=P, pre=P, dout=P, rows=10, Cin=8, Cout=8, act=2, p=0.0, rng=None, dtype=1, dx=P, dw=P, db=P, ws=P, size=1 << 30):
        return lib.affmae_linear_bwd(x, w, pre, dout, rows, Cin, Cout, act, p, rng, dtype, dx, dw, db, ws, size, None)

    assert bwd(dout=None) == -1 and bwd(dx=None, dw=None, db=None) == -1
    assert bwd(x=None) == -1 and bwd(w=None) == -1                # each needed for one of the gradients
    assert bwd(dw=None) == -1                                     # dbias comes with dweight
    assert bwd(pre=None) == -1                                    # an activation without the values in front of it
    assert bwd(p=0.2) == -1
    assert bwd(rows=0) == -2 and bwd(act=9) == -2 and bwd(p=1.5, rng=P) == -2
    for name in ("x", "w", "pre", "dout", "dx", "dw", "db"):
        assert bwd(**{name: P + 1}) == -2, name
    assert bwd(dtype=-1) == -3
    assert bwd(Cin=1 << 21) == -5
    need = lib.affmae_linear_bwd_workspace_bytes(10, 8, 8, 2, 0.0, 1, 1, 1)
    assert need >= 10 * 8 * 2                                     # dz
    assert bwd(ws=None) == -4 and bwd(size=need - 1) == -4 and bwd(ws=P + 64) == -4
    assert lib.affmae_linear_bwd_workspace_bytes(10, 0, 8, 2, 0.0, 1, 1, 1) == 0
    assert lib.affmae_linear_bwd_workspace_bytes(10, 8, 8, 2, 1.0, 1, 1, 1) == 0


def test_norm_refuses():
    lib = aff.load_library()

    def fwd(x=P, gamma=P, beta=P, B=2, N=16, C=8, G=2, eps=1e-5, act=0, dtype=1, out=P, mean=P, rstd=P, ws=P, size=1 << 30):
        return lib.affmae_norm_fwd(x, gamma, beta, B, N, C, G, eps, act, dtype, out, mean, rstd, ws, size, None)

    for name in ("x", "gamma", "beta", "out", "mean", "rstd"):
        assert fwd(**{name: None}) == -1, name
        assert fwd(**{name: P + 1}) == -2, name
    assert fwd(B=0) == -2 and fwd(N=0) == -2 and fwd(C=0) == -2 and fwd(G=0) == -2 and fwd(G=3) == -2
    assert fwd(eps=0.0) == -2 and fwd(eps=NAN) == -2 and fwd(eps=float("inf")) == -2 and fwd(act=7) == -2
    assert fwd(dtype=3) == -3
    assert fwd(C=1 << 21) == -5 and fwd(B=1 << 24, N=128) == -5 and fwd(B=1 << 24, N=1, G=2) == -5
    need = lib.affmae_norm_fwd_workspace_bytes(8, 16384, 64, 8, 1)
    if need:
        assert fwd(B=8, N=16384, C=64, G=8, ws=None, size=0) == -4 and fwd(B=8, N=16384, C=64, G=8, size=need - 1) == -4
    assert lib.affmae_norm_fwd_workspace_bytes(8, 16384, 64, 7, 1) == 0

    def bwd(x=P, gamma=P, beta=P, mean=P, rstd=P, dout=P, B=8, N=16384, C=64, G=8, act=0, dtype=1, dx=P, dg=P, db=P, ws=P, size=1 << 30):
        return lib.affmae_norm_bwd(x, gamma, beta, mean, rstd, dout, B, N, C, G, act, dtype, dx, dg, db, ws, size, None)

    for name in ("x", "gamma", "beta", "mean", "rstd", "dout", "dx", "dg", "db"):
        assert bwd(**{name: None}) == -1, name
        assert bwd(**{name: P + 1}) == -2, name
    assert bwd(gamma=None, beta=None) == -1                        # gradients of what is not there
    assert bwd(G=5) == -2 and bwd(act=-2) == -2 and bwd(dtype=9) == -3
    need = lib.affmae_norm_bwd_workspace_bytes(8, 16384, 64, 8, 1)
    if need:
        assert bwd(ws=None, size=0) == -4 and bwd(size=need - 1) == -4 and bwd(ws=P + 16) == -4
    assert lib.affmae_norm_bwd_workspace_bytes(0, 16384, 64, 8, 1) == 0


def test_dropout_refuses():
    lib = aff.load_library()

    def fwd(x=P, res=None, n=100, p=0.1, rng=P, dtype=1, out=P):
        return lib.affmae_dropout_fwd(x, res, n, p, rng, dtype, out, None)

    assert fwd(x=None) == -1 and fwd(out=None) == -1 and fwd(rng=None) == -1
    assert fwd(n=0) == -2 and fwd(n=-5) == -2 and fwd(p=1.0) == -2 and fwd(p=-1e-3) == -2 and fwd(p=NAN) == -2
    assert fwd(x=P + 1) == -2 and fwd(res=P + 1) == -2 and fwd(out=P + 1) == -2 and fwd(rng=P + 4) == -2
    assert fwd(dtype=5) == -3
    assert lib.affmae_dropout_bwd(None, 100, 0.1, P, 1, P, None) == -1
    assert lib.affmae_dropout_bwd(P, 100, 0.1, None, 1, P, None) == -1
    assert lib.affmae_dropout_bwd(P, 0, 0.1, P, 1, P, None) == -2


def test_binding_refuses_host_tensors_and_unknown_types():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        aff.affmae_linear_fwd(x, torch.zeros(8, 8))
    with pytest.raises(ValueError):
        aff.affmae_linear_bwd(x, torch.zeros(8, 8), x)
    with pytest.raises(ValueError):
        aff.affmae_norm_fwd(x[None], None, None)
    with pytest.raises(ValueError):
        aff.affmae_norm_bwd(x[None], None, None, x, x, x[None])
    with pytest.raises(ValueError):
        aff.affmae_dropout_fwd(x, 0.0)
    with pytest.raises(ValueError):
        aff.affmae_dropout_bwd(x, 0.0)
    with pytest.raises(ValueError):
        aff.affmae_dropout_fwd(x.half(), 0.0)


def test_activation_codes_of_header_and_binding():
    import os
    import re
    from paper_2602_16249_amd import binding
    text = open(os.path.join(os.path.dirname(aff.library_path()), "..", "include", "affmae.h")).read()
    codes = {name.lower(): int(v) for name, v in re.findall(r"AFFMAE_ACT_([A-Z]+) = (\d)", text)}
    assert codes == binding._ACTS
