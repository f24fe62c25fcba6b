"""CPU-side checks of the dense operators' binding: sizes that a C int does not hold are refused before the library sees their low 32 bits.
Tensors without storage stand for the ones on the device, and a library that is not to be called for the real one."""
import pytest
import torch

import paper_2602_16249_amd as aff
from paper_2602_16249_amd import binding

FAR = 2 ** 32  # its low 32 bits are 0


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


def _refused(call):
    with pytest.raises(aff.AffmaeError) as e:
        call()
    assert e.value.status == -5


@pytest.mark.parametrize("rows,cin,cout", [(FAR + 10, 1, 1), (10, FAR + 1, 1), (10, 1, FAR + 1), (2 ** 31, 1, 1)])
def test_linear_sizes(no_library, rows, cin, cout):
    x, w, dout = _meta(rows, cin), _meta(cout, cin), _meta(rows, cout)
    _refused(lambda: aff.affmae_linear_fwd(x, w))
    _refused(lambda: aff.affmae_linear_bwd(x, w, dout))
    _refused(lambda: aff.affmae_linear_bwd(x, None, dout, want_dx=False))
    _refused(lambda: aff.affmae_linear_bwd(None, w, dout, want_dweight=False))
    if rows > 10:
        lead = x.view(2, rows // 2, cin)  # several leading dimensions are as many rows
        _refused(lambda: aff.affmae_linear_fwd(lead, w))


@pytest.mark.parametrize("B,N,C,groups", [(1, FAR + 16384, 8, 1), (FAR + 2, 1, 8, 1), (1, 1, FAR + 8, 1), (2, 4, 8, FAR + 2), (2, 4, 8, 2 - FAR), (2 ** 31, 1, 1, 1)])
def test_norm_sizes(no_library, B, N, C, groups):
    x = _meta(B, N, C)
    stat = _meta(1, 1, dtype=torch.float32)
    _refused(lambda: aff.affmae_norm_fwd(x, None, None, groups))
    _refused(lambda: aff.affmae_norm_bwd(x, None, None, stat, stat, x, groups))
