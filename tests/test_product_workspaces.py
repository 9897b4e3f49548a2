"""Workspaces of the operators that are made of products: they hold what their copies write, and what they hold is bounded; sizes that no launch can have are refused (host functions: no GPU needed)."""
import pytest
import torch

import paper_2409_02208_amd as cbm
from paper_2409_02208_amd import binding

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


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("n,k,m", [(1024, (1 << 23) + 35 * 2048, 128), (1025, 1 << 24, 1000), (1024, 1 << 22, 512), (4096, (1 << 22) - 7, 64)])
def test_rows_of_four_million_values_and_more_are_not_copied(n, k, m, dtype):
    """Tiles that read whole units reach their rows by 32 bits from the first: 256 rows of 2^23 values are beyond them."""
    assert cbm.cbm_gated_linear_workspace_bytes(n, k, m, dtype) == 0
    assert cbm.cbm_linear_log_probs_workspace_bytes(n, k, 2 * m, dtype) <= 8 * n * _whole(2 * m, 128) + 4 * n + 32


FAR = 1 << 48  # between operands that are only addresses here


def _at(i):
    return (i + 1) * FAR


@pytest.mark.parametrize("type_", [0, 1, 2])
@pytest.mark.parametrize("n,k,m", [(1 << 31, 1, 64), (1 << 30, 8, 128), (1 << 24, 4, 1 << 14)])
def test_products_of_too_many_tiles_are_refused(n, k, m, type_):
    """2^24 tiles of 256 threads are as many threads as no launch has: an error before anything is launched."""
    lib = binding._lib()
    assert lib.cbm_gated_linear_workspace_bytes(n, k, m, type_) == 0
    assert lib.cbm_gated_linear(n, k, m, type_, 0, _at(0), k, _at(1), m, _at(2), m, _at(3), m, None, m, None, m, None, 0, None) == 5
    # X's gradient has as many with the sides the other way round
    assert lib.cbm_gated_linear_backward_workspace_bytes(n, 2 * m, k, type_) == 0
    assert lib.cbm_gated_linear_backward(n, 2 * m, k, type_, 0, _at(0), k, _at(1), 2 * m, _at(2), k, _at(3), k, _at(4), k, _at(5), k, _at(6), 2 * m, None, k, None, k, None, 0, None) == 5


@pytest.mark.parametrize("type_", [0, 1, 2])
@pytest.mark.parametrize("n,d,c", [(1 << 31, 8, 8), (1 << 30, 256, 2), (1 << 28, 8, 1024)])
def test_gradients_of_too_many_tiles_are_refused(n, d, c, type_):
    lib = binding._lib()
    assert lib.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, type_) == 0
    assert lib.cbm_linear_log_probs_backward(n, d, c, type_, _at(0), d, _at(1), c, _at(2), 64, _at(3), _at(4), _at(5), d, _at(6), c, None, 0, None) == 5
    assert lib.cbm_linear_log_probs_backward_workspace_bytes(1 << 20, d, c, type_) > 0
