"""Sizes of the workspaces of the operators between the products (host functions: no GPU needed)."""
import pytest

import paper_2409_02208_amd as cbm

PAIR = 2 * 4  # bytes of dgamma and dbeta of a column in a partial sum


@pytest.mark.parametrize("k", [1, 64, 1000, 3072 - 8, 3100, 12289, 16384, 16385, 40000, 1 << 17, 1 << 20, 1 << 24])
@pytest.mark.parametrize("n", [1, 100, 4096, 1 << 21])
def test_layer_norm_asks_for_the_partial_sums_that_a_shape_writes(n, k):
    """512 workgroups, 256 of the rows that half as many take (over 384 pieces of 16 bytes, of 16 bits 3,072 columns), and of rows too wide for registers 2,048 shares over a row's workgroups of
    256 pieces."""
    most = 512 if k <= 3072 else 256 if k <= 16384 else max(1, 2048 // -(-k // 2048))
    need = cbm.cbm_layer_norm_workspace_bytes(n, k)
    assert 0 < need <= min(n, most) * PAIR * k


def test_layer_norm_workspace_of_the_longest_rows_is_small_beside_them():
    n, k = 4096, 1 << 24
    assert cbm.cbm_layer_norm_workspace_bytes(n, k) <= n * k * 2 // 100


def test_none_for_sizes_that_are_refused():
    assert [cbm.cbm_layer_norm_workspace_bytes(n, k) for n, k in ((-1, 8), (8, 0), (8, -1), (8, (1 << 24) + 1), (0, 8))] == [0] * 5
