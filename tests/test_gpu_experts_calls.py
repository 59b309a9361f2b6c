"""What a caller of the layer of experts may hand over: ids without an expert, one workspace for calls of several sizes,
tensors that ask for gradients."""

import numpy as np
import pytest

from tests.test_gpu_experts import _cuda, _experts_case, _say, sd, torch  # noqa: F401  (the last two are fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E", [(2, 8), (40, 5), (300, 3)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_ids_past_the_last_expert_have_none(torch, sd, dtype, T, E):  # noqa: F811
    """An id of `experts` or more is a place without an expert, as a negative one is, for few slots and for many; its
    weight and what the workspace held do not matter."""
    H, F, k = 200, 150, 2
    args, host, _ = _experts_case(torch, sd, T, H, F, E, k, 0.5, seed=3)
    dt, routes = getattr(torch, dtype), args[2]
    ids, weight = host[3].copy(), host[4].copy()
    none = ids < 0
    assert none.any() and not none.all()
    ids[none] = np.resize([E, E + 1, 1 << 30, -2, 2**31 - 1, -(2**31)], none.sum())
    weight[none] = np.nan
    other = routes._replace(ids=_cuda(torch, ids.astype(np.int32)), weight=_cuda(torch, weight))
    ws = torch.full((sd.sdnn_experts_workspace_size(T, H, F, E, k, int(dt == torch.bfloat16)),), 255, dtype=torch.uint8,
                    device="cuda")
    _say("ids past the last", T, E, dtype)
    want = sd.experts_forward(*args, H, F, dtype=dt)
    assert torch.equal(sd.experts_forward(*args[:2], other, *args[3:], H, F, dtype=dt, ws=ws), want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_one_workspace_for_calls_of_several_sizes(torch, sd, dtype):  # noqa: F811
    """A workspace of the size for 9 tokens, which takes other kernels, for 1 to 9: same results as with one made for the
    call, nothing written past its end."""
    H, F, E, k = 130, 300, 24, 3
    dt = getattr(torch, dtype)
    need = sd.sdnn_experts_workspace_size(9, H, F, E, k, int(dt == torch.bfloat16))
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    for T in (9, 8, 1, 5):
        args, _, _ = _experts_case(torch, sd, T, H, F, E, k, 0.0)
        _say("one workspace", T, dtype)
        assert torch.equal(sd.experts_forward(*args, H, F, dtype=dt, ws=room[:need]), sd.experts_forward(*args, H, F, dtype=dt))
    assert bool((room[need:] == 255).all())
