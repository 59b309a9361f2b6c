"""What generates tokens, together: layers of experts, the norm, the 4-bit head and the choice of a token, as a program runs
them.

The step on a few rows and the layers on many compute the same: each layer rounds its input to 8 bits, where a difference of one
bfloat16 rounding (2^-9) moves about one code in twenty by a step of a sixteenth to an eighth, 1 to 2% of a layer's result, and
the result joins a row that is as large as itself.  Two layers of 5% each in the 2-norm bound that with room.
"""

import numpy as np
import pytest

from tests import generate_ref as gen
from tests.test_gpu_experts import _say, sd, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def _model(torch, seed, **sizes):  # noqa: F811
    from examples.generate import Model

    g = torch.Generator(device="cuda").manual_seed(seed)
    return Model(**{**dict(width=384, inner=200, experts=8, chosen=2, vocab=2000, layers=2), **sizes}, generator=g), g


@pytest.mark.parametrize("rows", [1, 7, 16])
def test_few_rows_and_many_are_the_same_layers(torch, sd, rows):  # noqa: F811
    model, g = _model(torch, 3)
    x = model.embedding[torch.randint(0, 2000, (rows,), generator=g, device="cuda")]
    _say("layers", rows)
    few, many = model.few(x).double(), model.many(x).double()
    assert float((few - many).norm() / many.norm()) <= 0.1


def test_head_and_tokens_from_the_definitions(torch, sd):  # noqa: F811
    """The logits of the 4-bit head against float64, and the tokens taken of them against the definition, row by row."""
    model, g = _model(torch, 4, vocab=20000)
    x = model.few(model.embedding[:9])
    z = sd.norm_quantize(x, model.gamma, normed=True)[3].double().cpu().numpy()
    w = gen.values4(*(t.view(torch.uint8).cpu().numpy() for t in (model.head, model.head_scale)), 384)
    _say("head and tokens")
    logits = model.logits(x)
    got = logits.double().cpu().numpy()
    assert np.all(np.abs(got - z @ w.T) <= (384 + 16) * 2.0 ** -24 * (np.abs(z) @ np.abs(w).T) + 2.0 ** -24 * np.abs(got))
    u = torch.rand(9, generator=g, device="cuda", dtype=torch.float64)
    k = torch.full((9,), 40, dtype=torch.int32, device="cuda")
    p = torch.full((9,), 0.9, device="cuda")
    taken = sd.sample(logits, u, top_k=k, top_p=p)
    for t in range(9):
        want = gen.sample(got[t], float(u[t]), 1.0, 40, float(np.float32(0.9)), 0.0)
        assert (int(taken.ids[t]), int(taken.kept[t])) == (want[0], want[2])


@pytest.mark.parametrize("places,vocab", [(1, 2000), (5, 33000), (16, 2000)])
def test_steps_of_a_graph_are_the_eager_ones(torch, sd, places, vocab):  # noqa: F811
    """A captured step replayed with new tokens, settings, random numbers and idle places: each equals the eager step on the
    same, and an idle place takes no token."""
    from examples.generate import Places

    model, g = _model(torch, 5, vocab=vocab)
    p = Places(model, places, g)
    p.tokens.copy_(torch.randint(0, vocab, (places,), generator=g, device="cuda"))
    p.capture()
    _say("steps", places, vocab)
    for i in range(5):
        p.live.copy_(torch.rand(places, generator=g, device="cuda") < (0.5 if i % 2 else 1.1))
        p.settings["temperature"].copy_(torch.rand(places, generator=g, device="cuda"))
        p.settings["top_k"].copy_(torch.randint(0, 30, (places,), generator=g, device="cuda"))
        before = p.tokens.clone()
        ids, prob = (t.clone() for t in p.next())
        p.tokens.copy_(before)
        want = p.step()
        assert torch.equal(ids, want[0]) and torch.equal(prob, want[1])
        assert bool((ids[~p.live] == -1).all()) and bool((ids[p.live] >= 0).all()) and bool((ids < vocab).all())
        p.tokens.copy_(torch.where(p.live, ids, p.tokens))
        torch.cuda.synchronize()


def test_example(torch, sd, capsys):  # noqa: F811
    import examples.generate as example

    taken = example.main(["--width", "256", "--inner", "128", "--experts", "8", "--chosen", "2", "--vocab", "3001", "--places",
                          "4", "--tokens", "6"])
    assert taken.shape == (6, 4) and bool((taken[:, 2:] == -1).all()) and bool((taken[:, :2] >= 0).all())
    assert "tokens/s" in capsys.readouterr().out


def test_example_with_one_place(torch, sd, capsys):  # noqa: F811
    """The only place generates."""
    import examples.generate as example

    taken = example.main(["--width", "256", "--inner", "128", "--experts", "8", "--chosen", "2", "--vocab", "3001", "--places",
                          "1", "--tokens", "6"])
    assert taken.shape == (6, 1) and bool((taken >= 0).all())
    assert " 0 tokens/s" not in capsys.readouterr().out


def test_tensors_of_two_devices_are_refused(torch, sd):  # noqa: F811
    """Tensors of two devices in one call are refused (here: a host tensor among those of the GPU)."""
    model, g = _model(torch, 6)
    x = model.embedding[:3]
    layer = model.layers[0]
    with pytest.raises(ValueError):
        sd.experts_layer(x, layer.gamma, model.routers[0].cpu(), 2, layer.w_in, layer.s_in, layer.w_out, layer.s_out, 200)
    with pytest.raises(ValueError):
        sd.sample(torch.zeros(2, 10, device="cuda"), torch.zeros(2, dtype=torch.float64))
    with pytest.raises(ValueError):
        sd.product_groups(x, model.head.cpu(), model.head_scale)


def test_first_calls_inside_a_capture(torch, sd):  # noqa: F811
    """In a process of its own, every call is made for the first time while a graph is captured: what a call sets up for its
    kernels does not end the capture, and the replay's results are the eager ones."""
    import os
    import subprocess
    import sys

    program = """
import torch, paper_1708_02937_amd as sd
g = torch.Generator(device="cuda").manual_seed(1)
x = torch.randn(5, 300, generator=g, device="cuda").bfloat16()
many = torch.randn(40, 300, generator=g, device="cuda")
w = torch.randn(70, 300, generator=g, device="cuda")
router = torch.randn(9, 300, generator=g, device="cuda") / 17
w_in, s_in = sd.quantize_blocks(torch.randn(9, 2, 130, 300, generator=g, device="cuda") / 17, 128)
w_out, s_out = sd.quantize_blocks(torch.randn(9, 300, 130, generator=g, device="cuda") / 11, 128)
gamma = torch.ones(300, device="cuda")
logits = torch.randn(3, 40000, generator=g, device="cuda")
u = torch.rand(3, generator=g, device="cuda", dtype=torch.float64)
p = torch.full((3,), 0.9, device="cuda")

def calls():
    q, s = sd.quantize_groups(w)
    return [sd.widen_groups(q, s, 300), sd.product_groups(x, q, s), sd.product_groups(many, q, s),
            *sd.experts_layer(x, gamma, router, 3, w_in, s_in, w_out, s_out, 130), *sd.sample(logits, u, top_p=p),
            *sd.sample(logits[:, :500], u, top_p=p)]

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = calls()
for _ in range(3):
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, calls()))
print("captured first")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    _say("first calls captured")
    done = subprocess.run([sys.executable, "-c", program], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "captured first" in done.stdout, done.stderr[-2000:]
