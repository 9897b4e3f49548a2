"""What the Python side of the operators that are made of products refuses before the library is called, and the sizes of their workspaces (no GPU needed)."""
import pytest
import torch

import paper_2409_02208_amd as cbm
from paper_2409_02208_amd import binding

x, w, h = torch.zeros((3, 6)), torch.zeros((6, 5)), torch.zeros((3, 5))
row = torch.zeros(3)
CALLS = {
    "cbm_gated_linear": (x, w, w, h),
    "cbm_gated_linear_backward": (h, x, w, w, h, h, x, w, w),
    "cbm_linear_log_probs": (x, w, None, row),
    "cbm_linear_log_probs_backward": (x, w, None, None, row, x, w),
    "cbm_orthogonalise": (x, x),
}


@pytest.mark.parametrize("name", CALLS)
def test_host_tensors_are_refused(name):
    with pytest.raises(ValueError, match="must be a 2-D device tensor"):
        getattr(cbm, name)(*CALLS[name], stream=0)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("what", [None, 3, "text", [[1.0]]])
def test_what_is_no_tensor_is_refused(name, what):
    with pytest.raises(ValueError, match="must be a tensor"):
        getattr(cbm, name)(what, *CALLS[name][1:], stream=0)


@pytest.mark.parametrize("name", CALLS)
def test_sparse_and_other_ranks_are_refused(name):
    first = CALLS[name][0]
    for t in (first.to_sparse(), first[0], first[None], first.to(torch.float64)):
        with pytest.raises(ValueError):
            getattr(cbm, name)(t, *CALLS[name][1:], stream=0)


@pytest.mark.parametrize("name", CALLS)
def test_streams_and_argument_counts(name):
    call = getattr(binding._calls(), name[len("cbm_"):])
    with pytest.raises(TypeError):
        call(*CALLS[name][:1])
    with pytest.raises(TypeError):
        getattr(cbm, name)(*CALLS[name], stream="a stream")


def test_activations_and_types_by_name():
    for bad in ("tanh", None, 0, []):
        with pytest.raises(ValueError, match="activation"):
            cbm.cbm_gated_linear(x, w, w, h, activation=bad, stream=0)
    for sizes, call in (((4, 5, 6), cbm.cbm_gated_linear_workspace_bytes), ((4, 5, 6), cbm.cbm_gated_linear_backward_workspace_bytes), ((4, 5, 6), cbm.cbm_linear_log_probs_workspace_bytes),
                        ((4, 5, 6), cbm.cbm_linear_log_probs_backward_workspace_bytes), ((4, 5), cbm.cbm_orthogonalise_workspace_bytes)):
        for bad in (torch.float64, torch.int32, "bf16", None):
            with pytest.raises(ValueError, match="is not one of"):
                call(*sizes, bad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_workspaces(dtype):
    size = torch.empty(0, dtype=dtype).element_size()
    for call in (cbm.cbm_gated_linear_workspace_bytes, cbm.cbm_gated_linear_backward_workspace_bytes, cbm.cbm_linear_log_probs_workspace_bytes, cbm.cbm_linear_log_probs_backward_workspace_bytes):
        assert [call(n, k, m, dtype) for n, k, m in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (4, 4, (1 << 24) + 1), (4, (1 << 24) + 1, 4))] == [0] * 5
    assert [cbm.cbm_orthogonalise_workspace_bytes(m, n, dtype) for m, n in ((0, 4), (4, 0), (-1, 4), (65537, 4))] == [0] * 4
    # what the scores of all classes would take is not asked for: dZ of a piece (512 MiB, or 1,024 classes), sums, shares
    n, d, c = 132534, 256, 128000
    assert 0 < cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, dtype) < n * c * size / 10
    assert 0 < cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, dtype) < n * c * size / 10
    # dG and dU of whole chunks, and shares of the weights' gradients
    need = cbm.cbm_gated_linear_backward_workspace_bytes(1000, 64, 100, dtype)
    assert need >= 2 * 1000 * 100 * size and need < 8 << 20
