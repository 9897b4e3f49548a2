"""The ReLU's backward pass from 8 bits where dY and dX share memory: in place with one stride, refused otherwise."""
import numpy as np
import pytest

from test_gpu_layer_norm import env  # noqa: F401

pytestmark = pytest.mark.gpu


def _kept(torch, cbm, n, k):
    x = torch.from_numpy(np.random.default_rng(n * k).standard_normal((n, k)).astype(np.float32)).cuda()
    Q, E = torch.empty((n, k), dtype=torch.int8, device="cuda"), torch.empty((n, (k + 31) // 32), dtype=torch.uint8, device="cuda")
    cbm.cbm_checkpoint_save(x, Q, E)
    return Q, E


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
def test_overlapping_gradients_are_refused(env, name):  # noqa: F811
    """Both matrices are valid by themselves: their strides are at least a row."""
    torch, cbm = env
    Q, E = _kept(torch, cbm, 4, 40)
    room = torch.arange(1000, device="cuda").to(getattr(torch, name))
    before = room.clone()
    view = lambda ld, at: room.as_strided((4, 40), (ld, 1), at)  # noqa: E731
    for dY, dX in ((view(48, 0), view(40, 0)), (view(40, 0), view(48, 0)), (view(48, 0), view(48, 1)), (view(48, 4), view(48, 0)), (view(40, 0), view(40, 120)),
                   (view(96, 0), view(96, 48))):  # the last: columns side by side in one buffer
        with pytest.raises(cbm.CbmError) as e:
            cbm.cbm_checkpoint_relu_backward(Q, E, dY, dX)
        assert e.value.status == 1
    torch.cuda.synchronize()
    assert torch.equal(room, before)
    cbm.cbm_checkpoint_relu_backward(Q, E, view(40, 0), view(40, 160))  # one behind the other
    assert torch.equal(room[160:320].view(4, 40), torch.where(Q > 0, before[:160].view(4, 40), torch.zeros_like(before[:160].view(4, 40))))


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("k", [1, 3, 5, 7, 9, 33, 36, 39, 47, 63, 65, 100, 255, 300, 500, 1001])
def test_in_place_is_what_it_is_elsewhere(env, name, k):  # noqa: F811
    """A row's last piece starts early: two lanes read and write what it shares with the piece before it, and gating twice is gating once, for infinities, NaN and both zeros, too."""
    torch, cbm = env
    n = 3000
    Q, E = _kept(torch, cbm, n, k)
    E[5, -1] = 255  # a block that is not finite
    gen = torch.Generator(device="cuda").manual_seed(k)
    dY = torch.randn((n, k + 3), device="cuda", generator=gen).to(getattr(torch, name))
    dY[::7, k - 1], dY[1::7, k - 1], dY[2::7, k - 1], dY[3::7] = float("nan"), float("inf"), -float("inf"), -0.0
    want = torch.empty_like(dY)
    cbm.cbm_checkpoint_relu_backward(Q, E, dY[:, :k], want[:, :k])
    behind = dY[:, k:].clone()
    cbm.cbm_checkpoint_relu_backward(Q, E, dY[:, :k], dY[:, :k])
    same = (dY[:, :k] == want[:, :k]) | (dY[:, :k].isnan() & want[:, :k].isnan())
    assert bool(same.all()) and torch.equal(dY[:, k:].nan_to_num(), behind.nan_to_num())
    block = slice((k - 1) // 32 * 32, k)
    assert bool(want[5, block].isnan().all())
