"""Workspaces of the operators that are made of products: they hold what their copies write, and what they hold is bounded (host functions: no GPU needed)."""
import pytest
import torch

import paper_2409_02208_amd as cbm

WIDE = [torch.bfloat16, torch.float16]


def _whole(v, of):
    return -(-v // of) * of


# Large 16-bit products.  Copies are written in whole groups of eight rows, so a k that is no multiple of eight has up to seven rows of zeros behind each copy of the weights; the first four sizes have no
# shares of K whose room would take them in.
SIZES = [(8192, 1537, 2049), (8147, 1734, 2285), (8192, 2047, 2047), (8869, 1634, 2496), (12001, 515, 4099), (1025, 1000, 25000), (4097, 512, 12288), (65535, 1023, 4095)]


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("n,k,m", SIZES)
def test_gated_layer_backward_has_room_for_whole_groups_of_rows(n, k, m, dtype):
    at, wide = _whole(m, 64), _whole(k, 8)
    slopes, x, weights = 2 * n * 2 * at, 2 * _whole(n, 8) * wide, 2 * 2 * wide * at
    assert cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, dtype) >= slopes + x + weights


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("n,k,m", SIZES)
def test_forward_passes_have_room_for_whole_groups_of_rows(n, k, m, dtype):
    wide = _whole(k, 8)
    assert cbm.cbm_gated_linear_workspace_bytes(n, k, m, dtype) >= 2 * _whole(n, 8) * wide + 2 * 2 * _whole(m, 32) * wide
    assert cbm.cbm_linear_log_probs_workspace_bytes(n, k, 2 * m, dtype) >= 2 * _whole(n, 8) * wide + 2 * _whole(2 * m, 8) * wide + 4 * n
    assert cbm.cbm_linear_log_probs_backward_workspace_bytes(n, k, 2 * m, dtype) >= 2 * _whole(n, 8) * wide + 2 * _whole(2 * m, 8) * wide + 2 * n * min(2 * m, 1024)


@pytest.mark.parametrize("dtype,type_", [(torch.float32, 0), (torch.bfloat16, 1), (torch.float16, 2)])
@pytest.mark.parametrize("n,d,c", [(2097152, 8, 131072), (65536, 8, 131072), (1 << 31, 8, 128), (300, 4, 1 << 24), (4096, 1024, 32000)])
def test_parts_of_rows_are_bounded(n, d, c, dtype, type_):
    """A maximum and a sum for 64 columns of a row (32 of up to 32 rows), 512 MiB at a time."""
    copies = 0 if type_ == 0 else 2 * _whole(n, 8) * _whole(d, 8) + 2 * _whole(c, 8) * _whole(d, 8)
    assert 0 < cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, dtype) <= (512 << 20) + 4 * n + 32 + copies
