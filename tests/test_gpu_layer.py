"""A layer of experts for a few tokens in one call, on an MI355X, against its 64-bit definition.

Tolerances, fixed before any run:
  * ids: equal (norm, logits and choice are fp64; they could differ only where choices lie within 1e-14 of each other);
    weights: one rounding to fp32, 2^-23 relative.
  * out, float32: the experts' bound of tests/test_gpu_experts.py (errors of p carried through, one step of a code of p where
    it lies that near to a boundary); a block's sum is weighted before it joins the total, one rounding more for each
    block and chosen expert; then s and the last sum, 2^-24 of each.
  * out, bfloat16: the same bound and the rounding of the result, 2^-8.
"""

import math

import numpy as np
import pytest

from tests import blocks_ref as ref
from tests.test_gpu_experts import _blocked, _cuda, _experts_ref, _hidden, _say, _to, sd, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

EPS = 1e-6


def _case(torch, sd, T, H, F, E, dtype, router, res, seed=0):  # noqa: F811
    """(tensors, their float64 values) of a layer."""
    rng = np.random.default_rng(T + 3 * H + 5 * F + 7 * E + seed)
    dt, rt = getattr(torch, dtype), getattr(torch, router)
    x, r = (_cuda(torch, _hidden(rng, (T, H)), dt) for _ in range(2))
    gamma = _cuda(torch, (1 + 0.1 * rng.standard_normal(H)).astype(np.float32))
    wr = _cuda(torch, rng.standard_normal((E, H)) / math.sqrt(H), rt)
    w1, s1, v1 = _blocked(torch, sd, rng.standard_normal((E, 2, F, H)) / math.sqrt(H), 128)
    w2, s2, v2 = _blocked(torch, sd, rng.standard_normal((E, H, F)) / math.sqrt(F), 128)
    bias = _cuda(torch, (0.1 * rng.standard_normal(E)).astype(np.float32))
    return dict(x=x, gamma=gamma, router=wr, w_in=w1, w_in_scale=s1, w_out=w2, w_out_scale=s2, inner=F,
                residual=r if res else None, bias=bias), (v1, v2)


def _want(args, values, k, live=None, score="softmax", bias=None, groups=1, kept=1, best=1, normalize=True, factor=1.0):
    """(out, bound, ids, weight) in 64 bits."""
    x = args["x"].double().cpu().numpy()
    r = None if args["residual"] is None else args["residual"].double().cpu().numpy()
    s, z = ref.norm(x, args["gamma"].cpu().numpy(), EPS, r)
    logits = z @ args["router"].double().cpu().numpy().T
    if live is not None:
        logits[~live] = -np.inf
    ids, weight = ref.route(logits, k, score, bias, groups, kept, best, normalize, factor)
    codes, scales = ref.quantize(z)
    v1, v2 = values
    out, tol = _experts_ref(ref.values(codes, scales, x.shape[1]), v1, v2, ids, weight, True)
    size, _ = _experts_ref(*(np.abs(v) for v in (ref.values(codes, scales, x.shape[1]), v1, v2)), ids, np.abs(weight), False)
    blocks = -(-args["inner"] // 128) * k
    tol = tol + (blocks + 20) * 2.0 ** -24 * np.abs(size) + 4 * 2.0 ** -24 * (np.abs(s) + np.abs(out))
    return s + out, tol, ids, weight


def _check(torch, got, want, dtype):  # noqa: F811
    out, tol, ids, weight = want
    assert np.array_equal(got.ids.cpu().numpy(), ids)
    assert np.all(np.abs(got.weight.double().cpu().numpy() - weight) <= 2.0 ** -23 * np.abs(weight) + 1e-45)
    half = 0.0 if dtype == "float32" else 2.0 ** -8
    off = np.abs(got.out.double().cpu().numpy() - out)
    assert np.all(off <= tol + half * (np.abs(out) + tol)), np.max(off / (tol + half * np.abs(out)))


def _run(sd, args, k, use_bias=True, **more):  # noqa: F811
    a = dict(args)
    a["bias"] = a["bias"] if use_bias else None
    return sd.experts_layer(a.pop("x"), a.pop("gamma"), a.pop("router"), k, **a, **more)


CASES = [
    # T, H, F, E, k, score, bias, groups, kept, best, normalize, factor, idle share
    (1, 256, 128, 4, 2, "softmax", False, 1, 1, 1, True, 1.0, 0.0),
    (1, 1, 1, 1, 1, "sigmoid", True, 1, 1, 1, False, 1.0, 0.0),
    (2, 130, 127, 8, 8, "softmax", True, 1, 1, 1, False, 2.5, 0.0),
    (3, 300, 70, 12, 3, "sigmoid", True, 4, 2, 2, True, 1.0, 0.0),
    (5, 129, 257, 5, 1, "softmax", False, 5, 3, 1, True, 1.0, 0.4),
    (9, 640, 200, 70, 6, "sigmoid", False, 7, 4, 2, False, 1.5, 0.2),
    (16, 500, 300, 6, 3, "softmax", True, 1, 1, 1, True, 1.0, 0.1),
    (16, 257, 600, 64, 8, "sigmoid", True, 8, 4, 2, True, 1.0, 0.0),
    (7, 128, 1030, 3, 3, "softmax", False, 1, 1, 1, True, 1.0, 0.0),
    (16, 64, 64, 2, 1, "softmax", False, 1, 1, 1, True, 1.0, 0.0),
    (4, 5000, 16, 3, 2, "softmax", False, 1, 1, 1, True, 1.0, 0.0),
    (6, 40, 30, 200, 20, "softmax", True, 2, 1, 2, True, 1.0, 0.3),
    (4, 96, 20, 64, 64, "sigmoid", True, 64, 64, 2, True, 1.0, 0.0),
    (2, 70, 50, 1024, 5, "sigmoid", False, 32, 3, 1, True, 1.0, 0.0),
    (3, 200, 100, 9, 4, "softmax", True, 1, 1, 1, True, 1.0, 1.0),
]


@pytest.mark.parametrize("T,H,F,E,k,score,bias,groups,kept,best,normalize,factor,idle", CASES)
@pytest.mark.parametrize("dtype,router", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("res", [False, True])
def test_layer(torch, sd, T, H, F, E, k, score, bias, groups, kept, best, normalize, factor, idle, dtype, router, res):  # noqa: F811
    args, values = _case(torch, sd, T, H, F, E, dtype, router, res)
    live = np.random.default_rng(T).random(T) >= idle
    b = args["bias"].cpu().numpy() if bias else None
    _say("layer", T, H, F, E, k, dtype, router, res)
    got = _run(sd, args, k, bias, score=score, groups=groups, groups_kept=kept, group_best=best, normalize=normalize,
               factor=factor, live=_cuda(torch, live) if idle else None)
    _check(torch, got, _want(args, values, k, live, score, b, groups, kept, best, normalize, factor), dtype)
    x = args["x"].double() + (args["residual"].double() if res else 0)
    dead = torch.from_numpy(~live).cuda()
    assert torch.equal(got.out[dead], x[dead].float().to(args["x"].dtype)) and bool((got.ids[dead] == -1).all())


@pytest.mark.parametrize("T", [1, 5, 16])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layer_is_the_separate_calls(torch, sd, T, dtype):  # noqa: F811
    """The norm, a product with the router in float64, the choice and the experts one by one: same experts and weights, and
    the same result up to the order of float sums."""
    H, F, E, k = 1000, 300, 16, 4
    args, _ = _case(torch, sd, T, H, F, E, dtype, "float32", True, seed=5)
    _say("layer and separate calls", T, dtype)
    got = _run(sd, args, k, score="sigmoid", groups=4, groups_kept=2, group_best=2)
    q, s, total, _ = sd.norm_quantize(args["x"], args["gamma"], EPS, residual=args["residual"])
    both = args["x"].double() + args["residual"].double()
    z = both / torch.sqrt((both * both).mean(1, keepdim=True) + EPS) * args["gamma"].double()
    logits = (z @ args["router"].double().t()).float()
    routes = sd.route(logits, k, "sigmoid", args["bias"], 4, 2, 2)
    assert torch.equal(routes.ids, got.ids)
    assert bool(((routes.weight - got.weight).abs() <= 1e-6 * got.weight).all())
    want = sd.experts_forward(q, s, routes, args["w_in"], args["w_in_scale"], args["w_out"], args["w_out_scale"], H, F,
                              dtype=torch.float32).double() + both
    # float32: codes of p that lie next to a boundary may move, one in 10^5 by a step of a sixteenth or less
    assert float((got.out.double() - want).norm() / want.norm()) <= (2e-5 if dtype == "float32" else 2.0 ** -8)


@pytest.mark.parametrize("T,H,F,E,k", [(5, 4200, 600, 16, 4), (16, 9000, 300, 20, 5), (1, 4097, 5000, 4, 2)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_wide_rows_of_many_experts(torch, sd, T, H, F, E, k, dtype):  # noqa: F811
    """Several turns of the width for several tiles of a workgroup: the same as the separate calls, to the tolerances of
    test_layer_is_the_separate_calls."""
    g = torch.Generator(device="cuda").manual_seed(H)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    x = rand(T, H).to(getattr(torch, dtype))
    gamma, router = 1 + 0.1 * rand(H), rand(E, H) / H ** 0.5
    w_in, s_in = sd.quantize_blocks(rand(E, 2, F, H) / H ** 0.5, 128)
    w_out, s_out = sd.quantize_blocks(rand(E, H, F) / F ** 0.5, 128)
    _say("layer wide", T, H, F, E, k, dtype)
    got = sd.experts_layer(x, gamma, router, k, w_in, s_in, w_out, s_out, F, eps=EPS)
    q, s, _, _ = sd.norm_quantize(x, gamma, EPS)
    z = x.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + EPS) * gamma.double()
    routes = sd.route((z @ router.double().t()).float(), k)
    assert torch.equal(routes.ids, got.ids)
    want = sd.experts_forward(q, s, routes, w_in, s_in, w_out, s_out, H, F, dtype=torch.float32).double() + x.double()
    assert float((got.out.double() - want).norm() / want.norm()) <= (2e-5 if dtype == "float32" else 2.0 ** -8)


def _rounded(v, bits):
    """float64 values rounded to `bits` bits, ties to even (normal values)."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


@pytest.mark.parametrize("T,H,F,E,k", [(1, 1000, 100, 8, 2), (6, 700, 200, 8, 3), (16, 513, 130, 5, 1)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_result_is_rounded_once(torch, sd, T, H, F, E, k, dtype):  # noqa: F811
    """Experts whose results are 2^-22 of the rows: what comes out is x + residual + theirs, in 64 bits, rounded once to its
    type.  (Theirs has the error of float sums, which decides only next to a middle: the rounding of both ends is allowed.)"""
    args, (v1, v2) = _case(torch, sd, T, H, F, E, dtype, "float32", True, seed=11)
    codes = args["w_out_scale"].view(torch.uint8)
    args["w_out_scale"] = torch.where(codes > 60, codes - 22, codes).view(torch.float8_e8m0fnu)  # but of empty blocks
    values = v1, v2 * 2.0 ** -22
    _say("layer rounded once", T, H, F, E, k, dtype)
    got = _run(sd, args, k)
    out, _, ids, weight = _want(args, values, k, bias=args["bias"].cpu().numpy())
    assert np.array_equal(got.ids.cpu().numpy(), ids)
    both = args["x"].double().cpu().numpy() + args["residual"].double().cpu().numpy()
    _, z = ref.norm(args["x"].double().cpu().numpy(), args["gamma"].cpu().numpy(), EPS, args["residual"].double().cpu().numpy())
    rows = ref.values(*ref.quantize(z), H)
    _, tol = _experts_ref(rows, *values, ids, weight, True)
    size, _ = _experts_ref(*(np.abs(v) for v in (rows, *values)), ids, np.abs(weight), False)
    tol = tol + (-(-F // 128) * k + 20) * 2.0 ** -24 * np.abs(size) + 2.0 ** -50 * np.abs(both)
    bits = 24 if dtype == "float32" else 8
    low, high = _rounded(out - tol, bits), _rounded(out + tol, bits)
    assert np.mean(low == high) > 0.5  # a code of p that may move takes a token's whole row of floats with it
    res = got.out.double().cpu().numpy()
    assert np.all((low <= res) & (res <= high)), int(np.sum((res < low) | (res > high)))


def test_rows_that_are_not_finite(torch, sd):  # noqa: F811
    """A row with an infinity or NaN has NaN logits: no expert takes it, its result is its sum, and the others do not
    notice; a router row of NaN is an expert that nobody takes, one with an infinity the expert of half the tokens."""
    T, H, F, E, k = 8, 200, 100, 6, 2
    args, values = _case(torch, sd, T, H, F, E, "float32", "float32", True)
    clean = _run(sd, args, k)
    bad = dict(args, x=args["x"].clone())
    bad["x"][2, 7], bad["x"][5, 199] = math.inf, math.nan
    _say("layer not finite")
    got = _run(sd, bad, k)
    keep = [0, 1, 3, 4, 6, 7]
    assert torch.equal(got.out[keep], clean.out[keep]) and torch.equal(got.ids[keep], clean.ids[keep])
    assert bool((got.ids[[2, 5]] == -1).all()) and not bool(got.weight[[2, 5]].any())
    sums = bad["x"] + bad["residual"]
    assert torch.equal(torch.nan_to_num(got.out[[2, 5]], 7.0, 8.0, 9.0), torch.nan_to_num(sums[[2, 5]], 7.0, 8.0, 9.0))
    sick = dict(args, router=args["router"].clone())
    sick["router"][3] = math.nan
    got = _run(sd, sick, k)
    assert not bool((got.ids == 3).any()) and bool((got.ids >= 0).all())
    sick["router"][3] = args["router"][3]
    sick["router"][3, 0] = math.inf
    got = _run(sd, sick, k, use_bias=False)
    up = (args["x"] + args["residual"])[:, 0] > 0
    assert torch.equal((got.ids == 3).any(1), up)
    assert bool((got.weight[up][:, 0] == 1).all()) and bool((got.ids[up][:, 0] == 3).all())


def test_zero_rows_and_ties(torch, sd):  # noqa: F811
    """A row of zeros has equal logits: the first experts take it, and its result is zero."""
    args, _ = _case(torch, sd, 3, 150, 90, 10, "bfloat16", "bfloat16", False)
    x = args["x"].clone()
    x[1] = 0
    _say("layer zeros")
    for score in ("softmax", "sigmoid"):
        got = _run(sd, dict(args, x=x), 4, use_bias=False, score=score)
        assert got.ids[1].tolist() == [0, 1, 2, 3] and not bool(got.out[1].any())
        assert bool((got.weight[1] == 0.25).all())


@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("E", [7, 64, 100])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_scores_of_unequal_logits(torch, sd, T, E, score):  # noqa: F811
    """Scores of 1 or 0 whose logits differ are equal: the lower expert is chosen, and the weights are theirs."""
    H, F, k = 64, 20, 5
    args, values = _case(torch, sd, T, H, F, E, "float32", "float32", False, seed=7)
    args["x"].fill_(1.0)
    args["gamma"].fill_(1.0)
    _say("layer equal scores", T, E, score)
    for levels in ((40, 60, 50, 70, 45, 41, -3), (-800, 5, -900, -760, -850, -870, -820), (0, -1, -2, 2, 1, 3, -3)):
        logits = [levels[(3 * e + e // 7) % 7] for e in range(E)]
        args["router"].copy_((torch.tensor(logits, dtype=torch.float32) / H)[:, None].expand(E, H))
        for normalize in (True, False):
            got = _run(sd, args, k, use_bias=False, score=score, normalize=normalize)
            _check(torch, got, _want(args, values, k, score=score, normalize=normalize), "float32")


def test_in_place_strides_and_workspace(torch, sd):  # noqa: F811
    """The output over x and over the residual, rows with strides at odd addresses, a workspace full of NaN of the size for
    16 tokens that serves smaller calls, and nothing written beside the results."""
    H, F, E, k = 330, 140, 7, 3
    need = sd.sdnn_experts_layer_workspace_size(16, H, F, E, k)
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    for T in (16, 1, 6):
        args, _ = _case(torch, sd, T, H, F, E, "bfloat16", "float32", True)
        want = _run(sd, args, k)
        _say("layer in place", T)
        got = _run(sd, args, k, ws=room[:need])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for name in ("x", "residual"):
            over = args[name].clone()
            got = _run(sd, {**args, name: over}, k, out=over, ws=room[:need])
            assert torch.equal(over, want.out) and got.out.data_ptr() == over.data_ptr()
        wide = {n: torch.full((T + 2, H + 9), 7.0, device="cuda", dtype=torch.bfloat16) for n in ("x", "residual", "out")}
        for n in ("x", "residual"):
            wide[n][1:T + 1, 3:3 + H] = args[n]
        far = torch.zeros(E, H + 5, device="cuda")
        far[:, 2:2 + H] = args["router"]
        part = {n: t[1:T + 1, 3:3 + H] for n, t in wide.items()}
        got = _run(sd, {**args, "x": part["x"], "residual": part["residual"], "router": far[:, 2:2 + H]}, k, out=part["out"])
        assert torch.equal(part["out"], want.out)
        part["out"].fill_(7.0)
        assert bool((wide["out"] == 7.0).all())
    assert bool((room[need:] == 255).all())


def test_empty_and_same_bits(torch, sd):  # noqa: F811
    args, _ = _case(torch, sd, 16, 512, 256, 12, "bfloat16", "bfloat16", True)
    _say("layer same bits")
    a = _run(sd, args, 4)
    for _ in range(5):
        assert all(torch.equal(u, v) for u, v in zip(a, _run(sd, args, 4)))
    got = _run(sd, dict(args, x=args["x"][:0], residual=None), 4)
    assert got.out.shape == (0, 512) and got.ids.shape == (0, 4) and got.weight.shape == (0, 4)
    one = [_run(sd, dict(args, x=args["x"][t:t + 1], residual=args["residual"][t:t + 1]), 4) for t in range(16)]
    assert torch.equal(torch.cat([o.ids for o in one]), a.ids) and torch.equal(torch.cat([o.weight for o in one]), a.weight)


def test_side_stream_and_graphs(torch, sd):  # noqa: F811
    """On another stream, and two captured layers of different sizes that share a workspace, replayed in turn with eager work
    between: each equals the eager result on that replay's inputs."""
    H, F, E, k = 384, 256, 8, 2
    layers = [_case(torch, sd, T, H, F, E, "bfloat16", "float32", True, seed=T)[0] for T in (1, 13)]
    ws = torch.empty(sd.sdnn_experts_layer_workspace_size(16, H, F, E, k), dtype=torch.uint8, device="cuda")
    want = _run(sd, layers[1], k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _say("layer streams")
    with torch.cuda.stream(side):
        got = _run(sd, dict(layers[1], x=(layers[1]["x"].float() * 2 / 2).bfloat16()), k)
    torch.cuda.synchronize()
    assert torch.equal(got.out, want.out)
    graphs, outs = [], []
    for args in layers:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(_run(sd, args, k, ws=ws))
    g = torch.Generator(device="cuda").manual_seed(4)
    for i in range(4):
        for args, graph, out in zip(layers, graphs, outs):
            args["x"].copy_(torch.randn(args["x"].shape, generator=g, device="cuda").bfloat16())
            want = _run(sd, args, k)
            graph.replay()
            assert all(torch.equal(u, v) for u, v in zip(out, want)), i
        torch.cuda.synchronize()


def test_two_streams_at_once(torch, sd):  # noqa: F811
    """Many calls on two streams at a time, each with a workspace of its own from the allocator."""
    H, F, E, k = 512, 384, 32, 4
    args, _ = _case(torch, sd, 16, H, F, E, "bfloat16", "float32", True)
    want = _run(sd, args, k)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    _say("layer two streams")
    outs = []
    for _ in range(20):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(_run(sd, args, k).out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want.out) for o in outs)


def test_arguments_are_checked(torch, sd):  # noqa: F811
    args, _ = _case(torch, sd, 3, 200, 100, 6, "float32", "float32", True)
    changes = [dict(x=args["x"][0]), dict(x=args["x"].double()), dict(x=args["x"].t()), dict(gamma=args["gamma"][:50]),
               dict(gamma=args["gamma"].bfloat16()), dict(router=args["router"][:, :100]), dict(router=args["router"].half()),
               dict(router=args["router"][:5]), dict(inner=99), dict(inner=0), dict(w_in=args["w_in"][:5]),
               dict(w_out_scale=args["w_out_scale"].cpu()), dict(residual=args["residual"].bfloat16()),
               dict(live=torch.ones(3, device="cuda")), dict(live=torch.ones(2, device="cuda", dtype=torch.bool)),
               dict(bias=torch.zeros(5, device="cuda")), dict(score="tanh"), dict(out=args["x"].bfloat16()),
               dict(ws=torch.empty(1 << 20, device="cuda")), dict(x=args["x"].clone().requires_grad_()),
               dict(router=args["router"].clone().requires_grad_())]
    for i, change in enumerate(changes):
        with pytest.raises(ValueError):
            _run(sd, {**args, **change}, 2)
            pytest.fail(f"case {i} was taken")
    for change, k, status in ((dict(), 7, 2), (dict(groups=4), 2, 2), (dict(eps=-1.0), 2, 2),
                              (dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda")), 2, 6)):
        with pytest.raises(sd.SdnnError) as e:
            _run(sd, {**args, **change}, k)
        assert e.value.status == status
    wide = dict(args, x=torch.ones(17, 200, device="cuda"), residual=None)
    with pytest.raises(sd.SdnnError, match="16 tokens"):
        _run(sd, wide, 2)
