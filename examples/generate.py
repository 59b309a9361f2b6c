"""Sequences generated with layers of experts: a batch of places, one token of each a step, from a captured graph.

A step is  x = embedding of the last tokens;  x = layer of experts (x) for each layer;  logits = norm(x) W_head;  tokens =
sample(logits)  at each place's own temperature, top-k, top-p and min-p.  The head's weights are 4 bits, the experts' 8.  A
place whose sequence has ended is idle: it takes part in no expert until a new sequence starts there.  A prompt's tokens go
through the same layers by the calls for any number of them.

    python examples/generate.py [--width 4096 --inner 1024 --experts 64 --chosen 8 --vocab 131072 --places 8 --layers 2]
"""

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1708_02937_amd as sd  # noqa: E402
from examples.experts_layer import ExpertsLayer, seconds  # noqa: E402


class Model:
    """An embedding, layers of experts, a norm and a head in 4 bits."""

    def __init__(self, width, inner, experts, chosen, vocab, layers, generator):
        rand = lambda *shape: torch.randn(*shape, generator=generator, device="cuda")  # noqa: E731
        self.width, self.vocab = width, vocab
        self.embedding = rand(vocab, width).bfloat16()
        self.layers = [ExpertsLayer(width, inner, experts, chosen, generator) for _ in range(layers)]
        self.routers = [layer.router.t().contiguous() for layer in self.layers]  # experts x width
        self.gamma = torch.ones(width, device="cuda")
        self.head, self.head_scale = sd.quantize_groups(rand(vocab, width) / width ** 0.5)

    def few(self, x, live=None):
        """The layers on up to 16 rows."""
        for layer, router in zip(self.layers, self.routers):
            x = sd.experts_layer(x, layer.gamma, router, layer.chosen, layer.w_in, layer.s_in, layer.w_out, layer.s_out,
                                 layer.inner, live=live, score="sigmoid", bias=layer.bias).out
        return x

    def many(self, x):
        """The layers on any number of rows, call by call."""
        for layer in self.layers:
            codes, scales, _, z = sd.norm_quantize(x, layer.gamma, normed=True)
            routes = sd.route(z.float() @ layer.router, layer.chosen, score="sigmoid", bias=layer.bias)
            x = sd.experts_forward(codes, scales, routes, layer.w_in, layer.s_in, layer.w_out, layer.s_out, self.width,
                                   layer.inner, residual=x)
        return x

    def logits(self, x):
        z = sd.norm_quantize(x, self.gamma, normed=True)[3]
        return sd.product_groups(z, self.head, self.head_scale, dtype=torch.float32)


class Places:
    """Generating sequences: the last token, the settings and the random numbers of each place, and the step on them."""

    def __init__(self, model, places, generator, temperature=0.8, top_k=50, top_p=0.95, min_p=0.02):
        full = lambda v: torch.full((places,), v, device="cuda")  # noqa: E731
        self.model, self.generator = model, generator
        self.tokens = torch.zeros(places, dtype=torch.int32, device="cuda")
        self.live = torch.ones(places, dtype=torch.bool, device="cuda")
        self.uniform = torch.zeros(places, dtype=torch.float64, device="cuda")
        self.settings = dict(temperature=full(temperature), top_k=full(top_k).int(), top_p=full(top_p), min_p=full(min_p))
        self.graph = None

    def step(self):
        x = self.model.embedding.index_select(0, self.tokens.clamp(min=0))
        taken = sd.sample(self.model.logits(self.model.few(x, self.live)), self.uniform, **self.settings)
        return torch.where(self.live, taken.ids, -1), taken.prob

    def capture(self):
        self.step()  # one-time set-up outside the capture
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.out = self.step()

    def next(self):
        """One step of the captured graph: the tokens it took (-1 at an idle place) and their shares."""
        self.uniform.copy_(torch.rand(self.uniform.shape, generator=self.generator, device="cuda", dtype=torch.float64))
        self.graph.replay()
        self.tokens.copy_(torch.where(self.live, self.out[0], self.tokens))
        return self.out


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("width", 4096), ("inner", 1024), ("experts", 64), ("chosen", 8), ("vocab", 131072), ("places", 8),
                        ("layers", 2), ("tokens", 32)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    model = Model(a.width, a.inner, a.experts, a.chosen, a.vocab, a.layers, g)
    places = Places(model, a.places, g)
    # a prompt ends in the first place: its last row goes on from there
    prompt = torch.randint(0, a.vocab, (100,), generator=g, device="cuda")
    rows = model.many(model.embedding[prompt])
    first = sd.sample(model.logits(rows[-1:]), torch.rand(1, generator=g, device="cuda", dtype=torch.float64),
                      temperature=torch.zeros(1, device="cuda"))
    places.tokens[:1] = first.ids
    places.live[(a.places + 1) // 2:] = False  # half of the places wait for a sequence
    places.capture()
    taken = torch.stack([places.next()[0].clone() for _ in range(a.tokens)])
    t = seconds(places.next, 50)
    print(f"{a.places} places: {t * 1e6:.0f} us a step from a graph, {int(places.live.sum()) / t:.0f} tokens/s; the first "
          f"sequence: {taken[:8, 0].tolist()}")
    return taken.cpu()


if __name__ == "__main__":
    start = time.perf_counter()
    main()
    print(f"{time.perf_counter() - start:.1f} s in all")
