"""The workspace of the norms' backward on the CPU: the sums of the channels take at most 2048 parts, however many images there are (8192 of
long ones)."""
import pytest

import paper_2602_16249_amd as aff


def _need(B, N, C, G, dtype):
    return aff.load_library().affmae_norm_bwd_workspace_bytes(B, N, C, G, dtype)


@pytest.mark.parametrize("dtype,el,limit", [(0, 4, 4096), (1, 2, 8192)])
def test_layer_norms_on_both_sides_of_the_row_kernels_limit(dtype, el, limit):
    for B in (1, 7, 300, 1024, 1025, 2049, 65536, 1 << 20):
        for C in (limit, limit + 1, limit + 2, limit + 4, limit + 8, 3 * limit):
            need = _need(B, 1, C, 1, dtype)
            # 2048 parts of two sums a channel; per image a pair of sums for each share of 256 columns or more, and their total
            assert 0 < need <= 2048 * 2 * C * 4 + 8 * B * (-(-C // 256) + 1) + 1024, (B, C)
        if B >= 65536:
            assert _need(B, 1, limit + 4, 1, dtype) <= B * (limit + 4) * el // 4


@pytest.mark.parametrize("B,N,C,G", [(20000, 2, 5000, 1), (65536, 2, 5000, 1), (65536, 7, 4200, 2), (9000, 3, 302, 2), (1 << 20, 3, 302, 2)])
def test_many_short_images(B, N, C, G):
    for dtype in (0, 1):
        assert _need(B, N, C, G, dtype) <= 2048 * 2 * C * 4 + 8 * B * G * (-(-C // G // 256) + 2) + 1024


@pytest.mark.parametrize("B,N,C,G", [(8192, 400, 256, 1), (8193, 400, 256, 1), (1 << 20, 64, 96, 3), (1 << 20, 33, 400, 1)])
def test_many_long_images(B, N, C, G):
    for dtype in (0, 1):
        assert _need(B, N, C, G, dtype) <= 8192 * 2 * C * 4 + 8 * B * G * 3 + 1024
