"""What the Python side of the operators between the products refuses before the library is called (host tensors will do: none of these calls gets that far)."""
import pytest
import torch

import paper_2409_02208_amd as cbm
from paper_2409_02208_amd import binding

f = torch.zeros((3, 40))
q, e = torch.zeros((3, 40), dtype=torch.int8), torch.zeros((3, 2), dtype=torch.uint8)
row = torch.zeros(3)

CALLS = {
    "cbm_layer_norm": (f, None, None, 1e-5, f),
    "cbm_layer_norm_backward": (f, f, None, row, row, f, None, None, None),
    "cbm_checkpoint_save": (f, q, e),
    "cbm_checkpoint_restore": (q, e, f),
    "cbm_checkpoint_relu_backward": (q, e, f, f),
    "cbm_checkpoint_weight_grad": (q, e, f, f, None),
    "cbm_log_probs": (f, None, None),
    "cbm_log_probs_backward": (f, None, row, None, row, None, f),
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
