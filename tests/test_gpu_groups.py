"""Matrices of 4 bits on an MI355X against their 64-bit definitions (tests/generate_ref.py).

Tolerances, fixed before any run:
  * codes, scales and widened values: equal.
  * product: K exact products (three parts of each where X is float) summed in fp32 in any order: (K + 16) 2^-24 of the sum
    of magnitudes, (3 K + 16) 2^-24 for float X (whose parts' magnitudes sum to 1.004 of the whole's), then one rounding to
    the result's type, 2^-24 or 2^-8 of the value.
"""

import math

import numpy as np
import pytest

from tests import generate_ref as gen
from tests.test_gpu_experts import _cuda, _hidden, _say, _to, sd, torch  # noqa: F401  (the last two are fixtures)

pytestmark = pytest.mark.gpu


def _matrix(torch, w):  # noqa: F811
    """(codes, scales) on the GPU from the reference's rounding, and their float64 values."""
    codes, scales = gen.quantize4(w)
    return (_cuda(torch, codes).view(torch.float4_e2m1fn_x2), _cuda(torch, scales).view(torch.float8_e8m0fnu),
            gen.values4(codes, scales, w.shape[1]))


def _bytes(torch, t):  # noqa: F811
    return t.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("rows,k", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 127), (4, 128), (7, 129), (33, 1001), (300, 4096)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_and_widen(torch, sd, rows, k, dtype):  # noqa: F811
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(rows * 5000 + k)
    x = _cuda(torch, _hidden(rng, (rows, k)), dt)
    _say("quantize_groups", rows, k, dtype)
    codes, scales = sd.quantize_groups(x)
    want, want_scales = gen.quantize4(x.double().cpu().numpy())
    assert np.array_equal(_bytes(torch, codes), want) and np.array_equal(_bytes(torch, scales), want_scales)
    exact = gen.values4(want, want_scales, k)
    for out in (torch.float32, torch.bfloat16):
        assert np.array_equal(sd.widen_groups(codes, scales, k, dtype=out).double().cpu().numpy(), exact)


def test_quantize_ties_and_extremes(torch, sd):  # noqa: F811
    """Every middle between two codes and its neighbours, at scales from the least to the largest; groups of zeros, of
    subnormal values, with infinities and NaN; each group alone."""
    middles = (gen.MAGNITUDES[1:] + gen.MAGNITUDES[:-1]) / 2
    base = np.concatenate([[6.0], middles, np.nextafter(middles.astype(np.float32), np.float32(9)),
                           np.nextafter(middles.astype(np.float32), np.float32(0)), -middles, gen.MAGNITUDES])
    base = np.resize(base, 64).astype(np.float32)
    rows = [base * np.float32(2.0) ** e for e in (-124, -60, -3, 0, 1, 50, 125)]
    rows += [np.zeros(64, np.float32), np.full(64, 1e-45, np.float32), np.full(64, 3.4028235e38, np.float32)]
    for bad in (np.inf, -np.inf, np.nan):
        row = base.copy()
        row[40] = bad
        rows.append(row)
    quiet = base.copy().view(np.uint32)
    quiet[3] = 0x7F800001  # a NaN whose bits are all in the lower half
    rows.append(quiet.view(np.float32))
    for top in (3.0, 6.0, np.nextafter(np.float32(6), np.float32(7)), np.nextafter(np.float32(3), np.float32(4))):
        row = np.zeros(64, np.float32)
        row[5] = top
        rows.append(row)
    x = np.stack(rows)
    _say("quantize_groups extremes")
    codes, scales = sd.quantize_groups(_cuda(torch, x))
    want, want_scales = gen.quantize4(x)
    assert np.array_equal(_bytes(torch, scales), want_scales)
    assert np.array_equal(_bytes(torch, codes), want)
    got = sd.widen_groups(codes, scales, 64, dtype=torch.float32).cpu().numpy()
    exact = gen.values4(want, want_scales, 64)
    with np.errstate(over="ignore"):
        assert np.array_equal(got, exact.astype(np.float32), equal_nan=True)


def test_quantize_below_the_normal_floats(torch, sd):  # noqa: F811
    """Groups at the least scale whose values are subnormal floats: codes to nearest even in steps of 2^-127, the middles and
    the floats beside them too; and matrices of random subnormal values."""
    middles = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * 2.0 ** -126
    top = np.float32(6 * 2.0 ** -126)
    middles = middles.astype(np.float32)
    base = np.concatenate([(gen.MAGNITUDES * 2.0 ** -126).astype(np.float32), middles, np.nextafter(middles, top),
                           np.nextafter(middles, np.float32(0))])
    x = np.zeros((4, 64), np.float32)
    x[0, :base.size], x[0, 32:32 + base.size] = base, -base
    x[1, :base.size], x[1, 5] = base, np.nextafter(top, np.float32(1))  # the next scale
    rng = np.random.default_rng(2)
    x[2] = rng.standard_normal(64) * 2.0 ** -126
    x[3] = rng.standard_normal(64) * 2.0 ** -130
    _say("quantize_groups subnormal")
    for dt in (torch.float32, torch.bfloat16):
        t = _cuda(torch, x).to(dt)
        codes, scales = sd.quantize_groups(t)
        want, want_scales = gen.quantize4(t.double().cpu().numpy())
        assert np.array_equal(_bytes(torch, scales), want_scales) and np.array_equal(_bytes(torch, codes), want)


def test_widen_every_code_and_scale(torch, sd):  # noqa: F811
    """All 256 scales over all 16 codes: subnormal values, ones past the float range, and NaN."""
    scales = np.arange(256, dtype=np.uint8).reshape(64, 4)
    codes = gen.pack4(np.tile(np.arange(16, dtype=np.uint8), (64, 8)))
    q, s = _cuda(torch, codes).view(torch.float4_e2m1fn_x2), _cuda(torch, scales).view(torch.float8_e8m0fnu)
    _say("widen_groups codes")
    exact = gen.values4(codes, scales, 128)
    with np.errstate(over="ignore"):
        want = exact.astype(np.float32)
    for out in (torch.float32, torch.bfloat16):
        got = sd.widen_groups(q, s, 128, dtype=out).float().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)


def test_stacks_strides_and_empty_matrices(torch, sd):  # noqa: F811
    rng = np.random.default_rng(4)
    x = _cuda(torch, _hidden(rng, (3, 5, 200)), torch.bfloat16)
    _say("quantize_groups stack")
    codes, scales = sd.quantize_groups(x)
    assert codes.shape == (3, 5, 128) and scales.shape == (3, 5, 8)
    flat, flat_scales = sd.quantize_groups(x.view(15, 200))
    assert np.array_equal(_bytes(torch, codes).reshape(15, -1), _bytes(torch, flat))
    assert np.array_equal(_bytes(torch, scales).reshape(15, -1), _bytes(torch, flat_scales))
    assert torch.equal(sd.widen_groups(codes, scales, 200).view(15, 200), sd.widen_groups(flat, flat_scales, 200))
    for off in (1, 3):  # rows at odd addresses, a stride that is no multiple of anything
        wide = _cuda(torch, _hidden(rng, (9, 307)), torch.float32)
        part = wide[:, off:off + 150]
        a, b = sd.quantize_groups(part), sd.quantize_groups(part.contiguous())
        assert all(np.array_equal(_bytes(torch, u), _bytes(torch, v)) for u, v in zip(a, b))
    none = sd.quantize_groups(torch.empty(0, 70, device="cuda"))
    assert none[0].shape == (0, 64) and sd.widen_groups(*none, 70).shape == (0, 70)
    assert sd.product_groups(torch.ones(2, 70, device="cuda"), *none).shape == (2, 0)
    assert sd.product_groups(torch.empty(0, 70, device="cuda"), *sd.quantize_groups(torch.ones(3, 70, device="cuda"))).shape == (0, 3)


def _bound(x, w, kind):
    k = x.shape[1]
    return ((3 * k if kind == "float32" else k) + 16) * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T)


@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (1, 17, 31), (2, 16, 33), (3, 100, 127), (1, 64, 128), (5, 65, 129), (16, 130, 500), (17, 33, 1000),
    (31, 200, 257), (32, 70, 1024), (33, 50, 1100), (64, 129, 640), (65, 40, 300), (130, 90, 200), (1, 300, 9000),
    (7, 20, 16384), (1, 8200, 70), (4, 9001, 260), (20, 8300, 40), (17, 2201, 1700), (33, 3001, 1300),
    (9, 60, 5000), (40, 300, 4500), (16, 8192, 600)])
@pytest.mark.parametrize("kinds", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"),
                                   ("float32", "bfloat16")])
def test_product(torch, sd, m, n, k, kinds):  # noqa: F811
    tx, ty = (getattr(torch, t) for t in kinds)
    rng = np.random.default_rng(m * 31 + n * 7 + k)
    x = _cuda(torch, _hidden(rng, (m, k)), tx)
    w, s, vals = _matrix(torch, rng.standard_normal((n, k)) / math.sqrt(k))
    b = _cuda(torch, rng.standard_normal(n).astype(np.float32))
    _say("product_groups", m, n, k, kinds)
    xv, bv = x.double().cpu().numpy(), b.double().cpu().numpy()
    z = xv @ vals.T
    off = _bound(xv, vals, kinds[0])
    half = 2.0 ** -24 if kinds[1] == "float32" else 2.0 ** -8
    for bias, ymax in ((None, None), (b, math.inf), (b, 0.75)):
        got = sd.product_groups(x, w, s, bias=bias, ymax=ymax, dtype=ty).double().cpu().numpy()
        want = z if bias is None else z + bv
        room = off if bias is None else off + 2.0 ** -24 * (np.abs(z) + np.abs(bv))
        if ymax is not None:
            want = np.clip(want, 0, ymax)
        assert np.all(np.abs(got - want) <= room + half * (np.abs(want) + room)), np.max(np.abs(got - want) - room)


def test_product_of_integers_is_exact(torch, sd):  # noqa: F811
    """Small integers sum exactly in any order, so every bit has to be right, at sizes that turn every loop."""
    rng = np.random.default_rng(8)
    for m, n, k in ((1, 4096, 4096), (16, 500, 3000), (40, 300, 2048), (64, 8200, 512), (48, 8190, 700), (64, 16380, 300),
                    (17, 9000, 650), (20, 16500, 300), (48, 16000, 300), (64, 20001, 300), (64, 33000, 300), (130, 9000, 300), (16, 9000, 1100), (3, 8300, 2100), (20000, 60, 200), (20000, 100, 200)):
        wv = rng.choice([-4.0, -2.0, 0.0, 1.0, 2.0, 3.0, 6.0], (n, k))
        wv[:, ::32] = 6.0  # scale 1
        xv = rng.integers(-8, 9, (m, k)).astype(np.float64)
        w, s, vals = _matrix(torch, wv[:64])
        assert np.array_equal(vals, wv[:64])
        w, s = sd.quantize_groups(_cuda(torch, wv, torch.float32))
        _say("product_groups integers", m, n, k)
        for dt in (torch.float32, torch.bfloat16):
            got = sd.product_groups(_cuda(torch, xv, dt), w, s, dtype=torch.float32)
            assert np.array_equal(got.double().cpu().numpy(), xv @ wv.T)


def test_product_of_floats_keeps_every_bit(torch, sd):  # noqa: F811
    """One product a row: 24-bit values, subnormal ones and the largest, times codes whose result a float holds."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal(40).astype(np.float32)
    x[:4] = [3.0e38, 1.0e-40, np.float32(2) ** -126 * 1.2345678, -1.1754942e-38]
    w = np.zeros((40, 40))
    w[np.arange(40), np.arange(40)] = np.where(np.arange(40) < 4, 1.0, rng.choice([0.5, 1.0, -2.0, 4.0], 40))
    codes, scale, _ = _matrix(torch, w)
    _say("product_groups bits")
    got = sd.product_groups(_cuda(torch, x[None]), codes, scale).cpu().numpy()[0]
    # The parts are bfloat16 values, whose least is 2^-133: what a float (a multiple of 2^-149)
    # has below that is less than 2^-133 and in no part.  Weights are 1 where that can be so.
    off = np.abs(got.astype(np.float64) - x.astype(np.float64) * np.diag(w))
    assert np.all(off[:4] < 2.0 ** -133) and off[0] == 0
    assert np.array_equal(got[4:], (x * np.diag(w).astype(np.float32))[4:])


def test_product_rows_and_weights_that_are_not_finite(torch, sd):  # noqa: F811
    """An infinity or NaN in one row reaches that row alone, a NaN group its output alone; NaN stays through the clamp."""
    rng = np.random.default_rng(6)
    for m in (3, 20, 50):
        for dt in (torch.float32, torch.bfloat16):
            x = _cuda(torch, rng.standard_normal((m, 300)), dt)
            wv = rng.choice([-1.0, 1.0, 2.0], (70, 300))
            w, s = sd.quantize_groups(_cuda(torch, wv, torch.float32))
            clean = sd.product_groups(x, w, s)
            y = x.clone()
            y[0, 299] = math.nan
            y[1, 5] = math.inf
            y[2, 130] = -math.inf
            _say("product_groups not finite", m, dt)
            got = sd.product_groups(y, w, s)
            assert bool(torch.isnan(got[0]).all()) and torch.equal(got[3:], clean[3:])
            assert np.array_equal(got[1].float().cpu().numpy(), np.inf * wv[:, 5])
            assert np.array_equal(got[2].float().cpu().numpy(), -np.inf * wv[:, 130])
            assert bool(torch.isnan(sd.product_groups(y, w, s, ymax=1.0)[0]).all())
            if dt == torch.float32:
                y = x.clone()
                y.view(torch.int32)[0, 7] = 0x7F800001  # a NaN whose bits are all in the lower half
                assert bool(torch.isnan(sd.product_groups(y, w, s)[0]).all())
            sick = s.clone()
            sick.view(torch.uint8)[33, 4] = 255
            got = sd.product_groups(x, w, sick)
            assert bool(torch.isnan(got[:, 33]).all())
            keep = torch.arange(70, device="cuda") != 33
            assert torch.equal(got[:, keep], clean[:, keep])


@pytest.mark.parametrize("m,n,k", [(1, 70, 300), (3, 70, 300), (20, 70, 300), (50, 70, 300), (5, 60, 2300), (64, 9000, 260), (4, 70, 9000)])
def test_product_of_infinite_weights(torch, sd, m, n, k):  # noqa: F811
    """A weight past the float range is infinite: an output with one is that infinity with the sign of x, NaN where x is 0,
    whatever bits x has and of whatever type it is; one with a finite weight of the same scale is its sum as ever."""
    rng = np.random.default_rng(m + n + k)
    wv = rng.choice([-1.0, 1.0, 2.0], (n, k))
    wv[:, 32:64] = 0.0  # one weight in the second group, each output its own
    code = np.resize([2, 3, 4, 6, -4, -6, 1.5, 1], n)  # the last two are finite
    wv[np.arange(n), 32 + np.arange(n) % 32] = code
    w, s = sd.quantize_groups(_cuda(torch, wv, torch.float32))
    assert np.array_equal(sd.widen_groups(w, s, k, dtype=torch.float32).cpu().numpy(), wv)
    # codes as for a scale of 1: 1 and 1.5 times 2^127 are floats, 2 times it is not
    index = np.zeros((n, 32), np.uint8)
    index[np.arange(n), np.arange(n) % 32] = gen.encode4(code)
    w.view(torch.uint8)[:, 16:32] = _cuda(torch, gen.pack4(index))
    s.view(torch.uint8)[:, 1] = 254
    inf = np.abs(code) >= 2
    x = rng.choice([1.0, 3.0, -0.5, 0.0, 2.0 ** -120, -1.0, 257.0], (m, k))
    x[:, 32:64][np.abs(x[:, 32:64]) > 1] = 1.0  # finite weights times these stay below the largest float
    x[0] = np.where(rng.random(k) < 0.5, 1.0, -1.0)
    some = rng.uniform(-1, 1, (m, k))
    for dt, rows in ((torch.float32, x), (torch.bfloat16, x), (torch.float32, some)):
        xt = _cuda(torch, rows, dt)
        xv = xt.double().cpu().numpy()
        _say("product_groups infinite weights", m, n, k, dt)
        got = sd.product_groups(xt, w, s, dtype=torch.float32).double().cpu().numpy()
        own = xv[:, 32 + np.arange(n) % 32]
        with np.errstate(invalid="ignore"):
            want = own * np.where(inf, np.copysign(np.inf, code), 1.0)
        assert np.array_equal(got[:, inf], want[:, inf], equal_nan=True)
        # the rest of a row (at most a few thousand) is below a rounding of 2^127 times 2^-120 and more, or is all there is
        values = wv.copy()
        values[:, 32:64] = 0.0
        values[np.arange(n), 32 + np.arange(n) % 32] = np.where(inf, 0.0, code * 2.0 ** 127)
        exact, room = xv @ values.T, _bound(xv, values, "float32")
        assert np.all(np.abs(got - exact)[:, ~inf] <= (room + 2.0 ** -24 * np.abs(exact))[:, ~inf])
    # what the rounding itself makes of the largest floats
    top = torch.full((2, 40), torch.finfo(torch.float32).max, device="cuda")
    got = sd.product_groups(torch.ones(m, 40, device="cuda"), *sd.quantize_groups(top))
    assert bool((got == math.inf).all())


def test_product_strides_outputs_and_streams(torch, sd):  # noqa: F811
    """Rows at any element address, an output inside a wider tensor whose rest stays, a side stream, and a graph that is
    replayed between eager calls."""
    rng = np.random.default_rng(12)
    w, s = sd.quantize_groups(_cuda(torch, rng.standard_normal((90, 333)), torch.float32))
    wide = _cuda(torch, rng.standard_normal((9, 700)), torch.bfloat16)
    for off in (0, 1, 5):
        part = wide[2:7, off:off + 333]
        _say("product_groups strides", off)
        want = sd.product_groups(part.contiguous(), w, s)
        room = torch.full((9, 101), 7.0, device="cuda", dtype=torch.bfloat16)
        got = sd.product_groups(part, w, s, out=room[1:6, 3:93])
        assert torch.equal(got, want) and got.data_ptr() == room[1:6, 3:93].data_ptr()
        room[1:6, 3:93] = 7.0
        assert bool((room == 7.0).all())
    x = wide[:4, :333].contiguous()
    want = sd.product_groups(x, w, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sd.product_groups(x, w, s)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sd.product_groups(x, w, s, ymax=math.inf)
    for i in range(4):
        x.copy_(wide[i:i + 4, 10:343])
        graph.replay()
        assert torch.equal(out, sd.product_groups(x, w, s, ymax=math.inf))
        torch.cuda.synchronize()


def test_offsets_past_32_bits(torch, sd):  # noqa: F811
    """Codes, dense values and a product's weights beyond 2^32 bytes into their tensors."""
    rows, k = 17000, 1 << 18  # 4.5e9 values, 2.2e9 bytes of codes
    _say("groups large")
    x = torch.zeros(rows, k, device="cuda", dtype=torch.bfloat16)
    last = torch.linspace(-6, 6, k, device="cuda").to(torch.bfloat16)
    x[-1] = last
    x[0] = -last
    codes, scales = sd.quantize_groups(x)
    for r, row in ((0, -last), (rows - 1, last)):
        c, t = sd.quantize_groups(row[None])
        assert torch.equal(codes[r].view(torch.uint8), c[0].view(torch.uint8))
        assert torch.equal(scales[r].view(torch.uint8), t[0].view(torch.uint8))
    del x
    y = sd.widen_groups(codes, scales, k)
    assert torch.equal(y[-1], sd.widen_groups(c, t, k)[0]) and torch.equal(y[0], -y[-1])
    assert not bool(y[rows // 2].any())
    del y
    codes2, scales2 = torch.cat([codes.view(torch.uint8)] * 2), torch.cat([scales.view(torch.uint8)] * 2)  # 4.5e9 bytes
    del codes, scales
    v = torch.ones(1, k, device="cuda", dtype=torch.bfloat16)
    v[:, : k // 2] = 0
    got = sd.product_groups(v, codes2.view(torch.float4_e2m1fn_x2), scales2.view(torch.float8_e8m0fnu), dtype=torch.float32)
    want = sd.product_groups(v, c, t, dtype=torch.float32)[0, 0]
    assert float(want) > 0
    for r, sign in ((0, -1), (rows - 1, 1), (rows, -1), (2 * rows - 1, 1)):
        assert float(got[0, r]) == sign * float(want)
    assert int((got != 0).sum()) == 4


def test_tensor_arguments_are_checked(torch, sd):  # noqa: F811
    x = torch.ones(4, 200, device="cuda")
    w, s = sd.quantize_groups(torch.ones(30, 200, device="cuda"))
    out = torch.empty(4, 30, device="cuda")
    calls = [
        lambda: sd.quantize_groups(x[0]), lambda: sd.quantize_groups(x.half()), lambda: sd.quantize_groups(x.t()),
        lambda: sd.quantize_groups(x.expand(3, 4, 200)), lambda: sd.widen_groups(w.view(torch.uint8), s, 200),
        lambda: sd.widen_groups(w, s[:20], 200), lambda: sd.widen_groups(w, s, 300), lambda: sd.widen_groups(w, s, 0),
        lambda: sd.widen_groups(w, s, 200, dtype=torch.float16), lambda: sd.product_groups(x[0], w, s),
        lambda: sd.product_groups(x[:, :100], w, s), lambda: sd.product_groups(x.double(), w, s),
        lambda: sd.product_groups(x, w[:20], s), lambda: sd.product_groups(x, w, s.cpu()),
        lambda: sd.product_groups(x, w, s, bias=torch.ones(29, device="cuda")),
        lambda: sd.product_groups(x, w, s, out=out.bfloat16()), lambda: sd.product_groups(x, w, s, out=out[:, ::2]),
        lambda: sd.product_groups(x, w, s, dtype=torch.float64), lambda: sd.product_groups(x.t(), w, s),
        lambda: sd.product_groups(x.clone().requires_grad_(), w, s), lambda: sd.quantize_groups(x.clone().requires_grad_()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"case {i} was taken")
    with pytest.raises(sd.SdnnError):
        sd.product_groups(x, w, s, ymax=0.0)
    with pytest.raises(TypeError):
        sd.product_groups(x, None, s)
