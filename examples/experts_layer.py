"""A layer of experts on 8-bit operands, served: a prompt, then single tokens from a captured graph.

One layer is  s = x + residual;  z = RMS norm of s;  experts = route(z W_router);  out = s + sum of the chosen experts'
gated networks on z in 8 bits.  The weights are rounded to 8 bits once; every call below is one of the library's, but
for the router's small product, which is the program's own.

    python examples/experts_layer.py [--width 4096 --inner 1024 --experts 64 --chosen 8 --prompt 2048 --layers 2]
"""

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1708_02937_amd as sd  # noqa: E402


class ExpertsLayer:
    """Weights of one layer: the norm's, the router's (float32), and the experts' in 8 bits."""

    def __init__(self, width, inner, experts, chosen, generator):
        def rand(*shape):
            return torch.randn(*shape, generator=generator, device="cuda") / shape[-1] ** 0.5

        self.width, self.inner, self.chosen = width, inner, chosen
        self.gamma = torch.ones(width, device="cuda")
        self.router = rand(experts, width).t().contiguous()
        self.bias = torch.zeros(experts, device="cuda")  # the balance bias, moved by whoever trains the router
        self.w_in, self.s_in = sd.quantize_blocks(rand(experts, 2, inner, width), 128)
        self.w_out, self.s_out = sd.quantize_blocks(rand(experts, width, inner), 128)

    def __call__(self, x, residual):
        codes, scales, total, z = sd.norm_quantize(x, self.gamma, residual=residual, normed=True)
        logits = z.float() @ self.router
        routes = sd.route(logits, self.chosen, score="sigmoid", bias=self.bias)
        out = sd.experts_forward(codes, scales, routes, self.w_in, self.s_in, self.w_out, self.s_out, self.width,
                                 self.inner, residual=None, dtype=x.dtype)
        return out, total  # the next layer adds them


def run(layers, x, residual):
    for layer in layers:
        x, residual = layer(x, residual)
    return x, residual


def capture(layers, x, residual):
    """A graph of the layers on these input tensors, and its outputs."""
    run(layers, x, residual)  # one-time set-up outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(layers, x, residual)
    return graph, out


def seconds(call, times):
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(times):
        call()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / times


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("width", 4096), ("inner", 1024), ("experts", 64), ("chosen", 8), ("prompt", 2048),
                        ("layers", 2)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    layers = [ExpertsLayer(a.width, a.inner, a.experts, a.chosen, g) for _ in range(a.layers)]

    prompt = torch.randn(a.prompt, a.width, generator=g, device="cuda").bfloat16()
    zero = torch.zeros_like(prompt)
    out, _ = run(layers, prompt, zero)
    t = seconds(lambda: run(layers, prompt, zero), 5)
    print(f"prompt of {a.prompt}: {t * 1e3:.2f} ms, {a.prompt / t:.0f} tokens/s")

    # single tokens: the same layers on one row, replayed from a graph; a row's result is the prompt's, up to rounding
    token, before = prompt[:1].clone(), zero[:1].clone()
    graph, (one, _) = capture(layers, token, before)
    graph.replay()
    torch.cuda.synchronize()
    far = float((one.float() - out[:1].float()).norm() / out[:1].float().norm())
    t = seconds(graph.replay, 50)
    print(f"one token: {t * 1e6:.1f} us from a graph, {seconds(lambda: run(layers, token, before), 50) * 1e6:.1f} us "
          f"call by call; its row differs from the prompt's by {far:.4f}")
    return far


if __name__ == "__main__":
    main()
