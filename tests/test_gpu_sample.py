"""The next token of each row on an MI355X against its 64-bit definition (tests/generate_ref.py).

ids and kept: equal.  Sums are carried in 64 bits on both sides, the kernel's of masses with 44 bits after the point: a decision
could differ where a share lies within 1e-11 of a token's end, relative to the row's mass.  No random row here comes that near
(each test says so), and rows made to lie on an end exactly have masses that are powers of two or equal ones.
prob: one rounding to fp32, and 1e-10 of the sums.
"""

import math

import numpy as np
import pytest

from tests import generate_ref as gen
from tests.test_gpu_experts import _cuda, _say, sd, torch  # noqa: F401  (the last two are fixtures)

pytestmark = pytest.mark.gpu


def _call(torch, sd, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, **more):  # noqa: F811
    f = lambda v: None if v is None else _cuda(torch, np.asarray(v, np.float32))  # noqa: E731
    return sd.sample(logits, _cuda(torch, np.asarray(u, np.float64)), f(temperature),
                     None if top_k is None else _cuda(torch, np.asarray(top_k, np.int32)), f(top_p), f(min_p), **more)


def _check(torch, sd, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, near=1e-11):  # noqa: F811
    """The call against the definition, row by row; returns what it gave."""
    got = _call(torch, sd, logits, u, temperature, top_k, top_p, min_p)
    l = logits.float().cpu().numpy().astype(np.float64)
    ids, prob, kept = (t.cpu().numpy() for t in got)
    for t in range(l.shape[0]):
        of = lambda v, none: none if v is None else float(np.float32(v[t]))  # noqa: E731
        want = gen.sample(l[t], float(u[t]), of(temperature, 1.0), 0 if top_k is None else int(top_k[t]), of(top_p, 1.0),
                          of(min_p, 0.0))
        assert near is None or want[3] > near, "a row too near to a boundary"
        assert (int(ids[t]), int(kept[t])) == (want[0], want[2]), (t, ids[t], kept[t], want)
        assert abs(prob[t] - want[1]) <= (2.0 ** -24 + 1e-10) * want[1] + 1e-45
    return got


def _logits(rng, T, V, banned=0.0):
    l = 2 * rng.standard_normal((T, V)) + 8 * rng.random((T, 1)) * (rng.random((T, V)) < 1e-3)
    return np.where(rng.random((T, V)) < banned, -np.inf, l)


def _settings(rng, T, mixed):
    off = rng.random((4, T)) < (0.35 if mixed else 0.0)
    return (np.where(off[0], rng.choice([0.0, 1.0], T), 0.3 + rng.random(T)), np.where(off[1], 0, rng.integers(1, 300, T)),
            np.where(off[2], 1.0, 0.5 + 0.49 * rng.random(T)), np.where(off[3], 0.0, 0.1 * rng.random(T)))


@pytest.mark.parametrize("T,V", [(1, 1), (5, 2), (9, 3), (20, 7), (33, 100), (40, 1001), (8, 4096), (7, 4097), (5, 20000),
                                 (4, 16384), (4, 16385), (3, 32768), (130, 32768), (6, 32769), (13, 50021), (3, 131072), (1, 262144), (140, 33000), (127, 33000),
                                 (260, 66000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("mixed,banned", [(False, 0.0), (True, 0.0), (True, 0.5)])
def test_sample(torch, sd, T, V, dtype, mixed, banned):  # noqa: F811
    rng = np.random.default_rng(T * 7 + V + int(mixed) + int(10 * banned))
    logits = _cuda(torch, _logits(rng, T, V, banned), getattr(torch, dtype))
    _say("sample", T, V, dtype, mixed, banned)
    _check(torch, sd, logits, rng.random(T), *_settings(rng, T, mixed))


@pytest.mark.parametrize("V", [50, 6000, 40000])
def test_each_setting_alone(torch, sd, V):  # noqa: F811
    """One filter at a time from next to nothing to next to everything, and all off."""
    rng = np.random.default_rng(V)
    T = 12
    logits = _cuda(torch, _logits(rng, T, V), torch.float32)
    _say("sample settings", V)
    for scale in (0.05, 1.0, 30.0):
        t = np.full(T, scale)
        _check(torch, sd, logits, rng.random(T), t)
        _check(torch, sd, logits, rng.random(T), t, top_k=np.linspace(1, V, T).astype(int))
        _check(torch, sd, logits, rng.random(T), t, top_k=[1, 2, 3, 5, 9, 20, 40, V // 2, 1024 % V, 1025 % V, V - 1, V + 5])
        _check(torch, sd, logits, rng.random(T), t, top_p=np.linspace(0.001, 0.999, T))
        _check(torch, sd, logits, rng.random(T), t, top_p=np.linspace(0.9, 0.9999, T), top_k=np.full(T, V - V // 3))
        _check(torch, sd, logits, rng.random(T), t, min_p=np.geomspace(1e-30, 1.0, T))
    _check(torch, sd, logits, rng.random(T))


@pytest.mark.parametrize("V", [64, 8192, 65536])
def test_equal_logits(torch, sd, V):  # noqa: F811
    """A flat row is the n-th of n equal shares; top_k and top_p cut among equal tokens by index; exact halves of the mass."""
    T = 9
    u = np.concatenate([[0.0, 0.5, 1 - 2.0 ** -53], (np.arange(6) + 0.5) / 6])
    flat = torch.full((T, V), 1.25, device="cuda")
    _say("sample equal", V)
    got = _call(torch, sd, flat, u)
    assert got.ids.tolist() == [int(x * V) for x in u] and bool((got.kept == V).all())
    for k in (1, 7, V // 2):
        got = _call(torch, sd, flat, u, top_k=[k] * T)
        assert got.ids.tolist() == [int(x * k) for x in u] and bool((got.kept == k).all())
    for share, n in ((0.25, V // 4), (0.5, V // 2), (0.75, 3 * V // 4)):
        got = _call(torch, sd, flat, u, top_p=[share] * T)
        assert bool((got.kept == n).all()) and got.ids.tolist() == [int(x * n) for x in u]
        got = _call(torch, sd, flat, u, top_p=[share] * T, top_k=[32] * T)
        assert bool((got.kept == 32 * share).all())
    assert bool((_call(torch, sd, flat, u, min_p=[1.0] * T).kept == V).all())
    # a few values: many tokens equal at every place where something is cut
    rng = np.random.default_rng(V)
    few = _cuda(torch, rng.integers(-3, 4, (T, V)) / 2.0, torch.bfloat16)
    _check(torch, sd, few, rng.random(T), top_k=np.linspace(1, V - 1, T).astype(int))
    _check(torch, sd, few, rng.random(T), top_p=np.linspace(0.1, 0.97, T), near=1e-13)
    _check(torch, sd, few, rng.random(T), np.full(T, 0.7), np.linspace(V // 3, V - 1, T).astype(int), np.linspace(0.1, 0.97, T),
           np.linspace(0, 0.3, T), near=1e-13)
    zeros = torch.zeros(T, V, device="cuda")
    zeros[:, ::2] = -0.0  # the same logit as 0
    assert _call(torch, sd, zeros, u, top_k=[8] * T).ids.tolist() == [int(x * 8) for x in u]
    assert bool((_call(torch, sd, zeros, u, [0.0] * T).ids == 0).all())


@pytest.mark.parametrize("V", [70000, 131072])
def test_nearly_flat_rows(torch, sd, V):  # noqa: F811
    """Every logit in one bucket, and all different: the list does not hold them, and the row is searched."""
    rng = np.random.default_rng(V)
    T = 5
    logits = _cuda(torch, (3 + 0.03 * rng.random((T, V))), torch.float32)
    _say("sample nearly flat", V)
    _check(torch, sd, logits, rng.random(T), top_p=np.linspace(0.1, 0.9, T), near=1e-13)
    _check(torch, sd, logits, rng.random(T), top_k=[1, 100, 1024, 5000, V - 2])
    _check(torch, sd, logits, rng.random(T), None, [40, 1024, 20000, 60000, 0], [0.5, 0.3, 0.9, 0.99, 0.2],
           [0.0, 0.99, 0.98, 0.0, 0.999], near=1e-13)
    for V in (16000, 30000):  # one launch, and four
        _check(torch, sd, logits[:, :V], rng.random(T), None, [40, 1024, 9000, 0, 0], [0.5, 0.3, 0.9, 0.99, 0.2], near=1e-13)


@pytest.mark.parametrize("T,V", [(6, 5000), (6, 40000), (150, 40000), (160, 40000), (2, 300000)])
def test_few_tokens_kept_of_uneven_rows(torch, sd, T, V):  # noqa: F811
    """top_k where the tokens that count lie together, in a few runs, or at even distances; where keys span all that floats
    can; where many are equal; and around as many tokens as half the runs of 8 or 64 tokens that a row has."""
    rng = np.random.default_rng(T + V)
    _say("sample uneven", T, V)
    at = np.arange(V)
    base = 2 * rng.standard_normal((T, V))
    rows = {
        "banned but a run": np.where((at >= V // 3) & (at < V // 3 + 900), base, -np.inf),
        "banned but a few": np.where(at % 97 == 5, base, -np.inf),
        "banned but 70": np.where((at >= 64) & (at < 134), base, -np.inf),
        "in order": np.broadcast_to(-at * (40.0 / V), (T, V)),
        "against the order": np.broadcast_to(at * (40.0 / V), (T, V)),
        "the best together": base + 30.0 * (at // 256 == 7),
        "far apart": np.where(rng.random((T, V)) < 0.5, base, -3e38 * rng.random((T, V))),
        "one far above": base + 1e30 * (at == V // 2),
        "few values": np.round(base),
        "subnormal": base * 1e-40,
    }
    k = np.resize([1, 2, 50, 64, 69, 70, 71, 128, 200, 256, 257, 312, 320, 400, 513, 900, 1024, 1025], T)
    for name, l in rows.items():
        logits = _cuda(torch, l, torch.float32)
        for first in range(1 if T > 100 else 3):
            near = None if name in ("in order", "against the order", "few values") else 1e-11
            _check(torch, sd, logits, rng.random(T), top_k=np.roll(k, 5 * first)[:T], near=near)
            _check(torch, sd, logits, rng.random(T), np.full(T, 0.7), np.roll(k, 6 * first + 1), np.full(T, 0.83), near=near)


@pytest.mark.parametrize("V", [300, 40000])
def test_rows_without_tokens_and_not_finite(torch, sd, V):  # noqa: F811
    rng = np.random.default_rng(1)
    l = _logits(rng, 10, V).astype(np.float32)
    l[0] = -np.inf
    l[1] = np.nan
    l[2, :] = -np.inf
    l[2, V - 1] = -3e38  # one token, the least of all
    l[3, 5:9] = np.inf  # these share the row
    l[4, ::2] = np.nan
    l[5] = np.where(np.arange(V) % 3 == 0, 3e38, -3e38)
    l[6] = 1e-44 * (np.arange(V) % 5)  # subnormal
    u = rng.random(10)
    logits = _cuda(torch, l)
    _say("sample not finite", V)
    got = _check(torch, sd, logits, u)
    assert got.ids[:3].tolist() == [-1, -1, V - 1] and got.kept[:3].tolist() == [0, 0, 1] and int(got.ids[3]) == 5 + int(4 * u[3])
    for settings in _settings(rng, 10, True), _settings(rng, 10, False), ([0.0] * 10, None, None, None):
        _check(torch, sd, logits, u, *settings, near=None)
    got = _check(torch, sd, logits, u, top_k=[2] * 10)
    assert got.kept[:4].tolist() == [0, 0, 1, 2] and int(got.ids[3]) == 5 + int(2 * u[3])


@pytest.mark.parametrize("V", [200, 40000])
def test_settings_at_their_limits(torch, sd, V):  # noqa: F811
    rng = np.random.default_rng(2)
    temperature = [0.0, -1.0, math.nan, 1e-45, 1e-30, 1e30, math.inf, 3e38, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0]
    T = len(temperature)
    logits = _cuda(torch, _logits(rng, T, V), torch.float32)
    u = rng.random(T)
    _say("sample limits", V)
    _check(torch, sd, logits, u, temperature, near=None)
    best = logits.argmax(1)
    got = _call(torch, sd, logits, u, temperature)
    assert torch.equal(got.ids[:5].long(), best[:5]) and got.kept[:3].tolist() == [1, 1, 1]
    top_p = [0.0, -1.0, 1e-45, math.nan, 2.0, math.inf, 1 - 2.0 ** -24, 0.5, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0]
    min_p = [0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, math.nan, -1.0, 1.0, 5.0, math.inf, 1e-45, 1e-30]
    top_k = [0, -5, 1, 2**31 - 1, -(2**31), V, V - 1, V + 1, 0, 0, 0, 0, 0, 3, 0]
    got = _check(torch, sd, logits, u, None, top_k, top_p, min_p)
    assert got.kept[:3].tolist() == [1, 1, 1] and got.kept[10:13].tolist() == [1, 1, 1]
    for edge in (0.0, 1 - 2.0 ** -53):  # the first and the last of the kept tokens
        got = _call(torch, sd, logits, [edge] * T, top_k=[7] * T)
        seven = torch.topk(logits, 7, dim=1).indices
        assert torch.equal(got.ids.long(), seven.amin(1) if edge == 0 else seven.amax(1))


@pytest.mark.parametrize("V", [1000, 45000])
def test_every_uniform_number(torch, sd, V):  # noqa: F811
    """One row drawn at many uniform numbers: the inverse of its distribution function, every kept token in its turn."""
    rng = np.random.default_rng(9)
    T = 1500
    l = _logits(rng, 1, V).astype(np.float32)
    u = np.sort(rng.random(T))
    logits = _cuda(torch, l).expand(T, V).contiguous()
    _say("sample distribution", V)
    got = _call(torch, sd, logits, u, top_k=[60] * T, top_p=[0.95] * T)
    want = [gen.sample(l[0].astype(np.float64), x, 1.0, 60, float(np.float32(0.95)), 0.0) for x in u]
    assert got.ids.tolist() == [w[0] for w in want] and bool((got.kept == want[0][2]).all())
    assert bool((got.ids[1:] >= got.ids[:-1]).all()) and len(set(got.ids.tolist())) > 10


@pytest.mark.parametrize("T,V,k", [(64, 40000, 600), (64, 40000, 1000), (64, 131072, 1024), (64, 131072, 5000), (3, 131072, 1000),
                                   (40, 40000, 5000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_last_kept_token_before_dropped_ones(torch, sd, T, V, k, dtype):  # noqa: F811
    """Numbers next to 1 take the last kept token, also where the row's last quarter holds many tokens just below the cut and
    none that is kept: sums over those add nothing, whatever their rounding.  The least kept mass is above e^-12 of the row's
    first and more than 1e-9 of all (5000 at the most); u leaves 2^-51 of all at the most, and sums are off by some 2^-50: the
    last kept token is the first whose sum exceeds u."""
    rng = np.random.default_rng(T + V + k)
    l = 2 * rng.standard_normal((T, V))
    at = 3 * V // 4
    cut = np.sort(l[:, :at], axis=1)[:, -k]
    l[:, at:] = -40.0
    for t in range(T):
        some = at + rng.choice(V - at, 400, replace=False)
        l[t, some] = cut[t] - 0.02 * (1 + rng.random(400))
    logits = _cuda(torch, l, getattr(torch, dtype))
    l = logits.float().cpu().numpy().astype(np.float64)
    _say("sample last kept", T, V, k, dtype)
    for u in (1 - 2.0 ** -53, 1 - 2.0 ** -52, 1 - 2.0 ** -51):
        got = _call(torch, sd, logits, [u] * T, top_k=[k] * T)
        order = [np.lexsort((np.arange(V), -l[t]))[:k] for t in range(T)]
        assert bool((got.kept == k).all()) and bool((got.prob > 0).all())
        assert got.ids.tolist() == [int(o.max()) for o in order]


def test_strides_workspace_streams_and_graphs(torch, sd):  # noqa: F811
    """Rows at odd addresses inside a wider tensor, a workspace of the size for 9 rows full of ones for fewer, a side stream,
    and captured calls of different sizes that share a workspace, replayed with eager work between."""
    rng = np.random.default_rng(5)
    V = 40000
    need = sd.sdnn_sample_workspace_size(9, V)
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    wide = _cuda(torch, _logits(rng, 11, V + 50), torch.bfloat16)
    _say("sample strides")
    for T in (9, 1, 4, 9):
        settings = _settings(rng, T, True)
        u = rng.random(T)
        part = wide[1:1 + T, 3:3 + V]
        a = _call(torch, sd, part, u, *settings, ws=room[:need])
        b = _call(torch, sd, part.contiguous(), u, *settings)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        _check(torch, sd, part.contiguous(), u, *settings)
    assert bool((room[need:] == 255).all())
    logits = wide[:6, :V].contiguous()
    u = _cuda(torch, rng.random(6))
    k = torch.full((6,), 50, device="cuda", dtype=torch.int32)
    p = torch.full((6,), 0.9, device="cuda")
    want = sd.sample(logits, u, top_k=k, top_p=p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sd.sample(logits, u, top_k=k, top_p=p)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    calls = [lambda ws: sd.sample(logits, u, top_k=k, top_p=p, ws=ws), lambda ws: sd.sample(logits[:2], u[:2], top_p=p[:2], ws=ws),
             lambda ws: sd.sample(logits[:, :900], u, top_k=k, ws=ws)]
    graphs, outs = [], []
    for call in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(call(room[:need]))
    g = torch.Generator(device="cuda").manual_seed(3)
    for i in range(4):
        u.copy_(torch.rand(6, generator=g, device="cuda", dtype=torch.float64))
        logits.copy_((2 * torch.randn(6, V, generator=g, device="cuda")).bfloat16())
        for call, graph, out in zip(calls, graphs, outs):
            graph.replay()
            want = call(None)
            assert all(torch.equal(x, y) for x, y in zip(out, want)), i
        torch.cuda.synchronize()


def test_many_rows_and_offsets_past_32_bits(torch, sd):  # noqa: F811
    rows, V = 65000, 66200  # 4.3e9 logits
    _say("sample large")
    logits = torch.zeros(rows, V, device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(3)
    some = [0, 1, rows // 2, rows - 2, rows - 1]
    logits[some] = (3 * torch.randn(5, V, generator=g, device="cuda")).bfloat16()
    u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
    k = torch.full((rows,), 40, device="cuda", dtype=torch.int32)
    got = sd.sample(logits, u, top_k=k)
    few = sd.sample(logits[some], u[some], top_k=k[:5])
    assert all(torch.equal(a[some], b) for a, b in zip(got, few))
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[some] = False
    assert torch.equal(got.ids[rest].long(), (u[rest] * 40).long())


def test_arguments_are_checked(torch, sd):  # noqa: F811
    logits, u = torch.randn(4, 50, device="cuda"), torch.rand(4, device="cuda", dtype=torch.float64)
    one, k = torch.ones(4, device="cuda"), torch.ones(4, device="cuda", dtype=torch.int32)
    calls = [lambda: sd.sample(logits[0], u), lambda: sd.sample(logits.double(), u), lambda: sd.sample(logits.t(), u),
             lambda: sd.sample(logits, u.float()), lambda: sd.sample(logits, u[:3]), lambda: sd.sample(logits, u.cpu()),
             lambda: sd.sample(logits, u, temperature=one[:3]), lambda: sd.sample(logits, u, temperature=k),
             lambda: sd.sample(logits, u, top_k=one), lambda: sd.sample(logits, u, top_k=k.long()),
             lambda: sd.sample(logits, u, top_p=one.double()), lambda: sd.sample(logits, u, min_p=one.cpu()),
             lambda: sd.sample(logits.clone().requires_grad_(), u), lambda: sd.sample(logits, u, ws=one)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"case {i} was taken")
    with pytest.raises(TypeError):
        sd.sample(logits, u, temperature=0.7)
    wide = torch.randn(2, 40000, device="cuda")
    with pytest.raises(sd.SdnnError) as e:
        sd.sample(wide, u[:2], ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 6
    got = sd.sample(logits[:0], u[:0])
    assert got.ids.shape == (0,) and got.kept.shape == (0,)
