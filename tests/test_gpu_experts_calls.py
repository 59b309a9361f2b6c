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


def test_inputs_that_ask_for_gradients_are_refused(torch, sd):  # noqa: F811
    """The layer has no gradients: an input that requires one is a ValueError while gradients are recorded, and so is one
    with a tangent; results are not silently cut off from it.  Under no_grad and inference_mode, and detached, the same
    tensors are ordinary inputs."""
    x, gamma = torch.randn(6, 200, device="cuda"), torch.ones(200, device="cuda")
    logits, bias = torch.randn(6, 8, device="cuda"), torch.zeros(8, device="cuda")
    a, sa = sd.quantize_blocks(x)
    w, sw = sd.quantize_blocks(torch.randn(70, 200, device="cuda"), 128)
    routes = sd.route(logits, 2)
    w_in, s_in = sd.quantize_blocks(torch.randn(8, 2, 40, 200, device="cuda"), 128)
    w_out, s_out = sd.quantize_blocks(torch.randn(8, 200, 40, device="cuda"), 128)
    out_bias = torch.zeros(70, device="cuda")

    def experts(weight, residual):
        return sd.experts_forward(a, sa, routes._replace(weight=weight), w_in, s_in, w_out, s_out, 200, 40,
                                  residual=residual, dtype=torch.float32)

    calls = [
        (lambda t: sd.quantize_blocks(t), x), (lambda t: sd.norm_quantize(t, gamma), x),
        (lambda t: sd.norm_quantize(x, t), gamma), (lambda t: sd.norm_quantize(x, gamma, residual=t), x),
        (lambda t: sd.norm_quantize(x, gamma, residual=x, out_sum=t), x.clone()), (lambda t: sd.route(t, 2), logits),
        (lambda t: sd.route(logits, 2, bias=t), bias),
        (lambda t: sd.product_blocks(a, sa, w, sw, 200, bias=t), out_bias),
        (lambda t: sd.product_blocks(t, sa, w, sw, 200), a), (lambda t: experts(t, None), routes.weight),
        (lambda t: experts(routes.weight, t), x),
    ]
    for i, (call, t) in enumerate(calls):
        _say("gradient", i)
        asks = t.detach().clone().requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call(asks)
            pytest.fail(f"case {i} was taken")
        call(asks.detach())
        with torch.no_grad():
            call(asks)
        with torch.inference_mode():
            call(asks)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(ValueError, match="gradient"):
            sd.norm_quantize(dual, gamma)
