"""The operators of a layer of experts on an MI355X against their 64-bit definitions (tests/blocks_ref.py).

Tolerances, fixed before any run:
  * codes, scales, sums and normed rows: equal.  The kernel carries them in fp64 and rounds once, the definition too;
    they could differ only where a value lies within 1e-15 of a rounding boundary.
  * ids, offsets, order: equal; weights: one rounding to fp32, 2^-23 relative.
  * fp32 product: K products summed in fp32 in any order, (K + 16) 2^-24 of the sum of magnitudes.
  * bfloat16 product: the output's rounding, 2^-8 of the value, and what the 8-bit matrix instructions drop: they add
    groups of at most 32 products aligned to the group's largest with 14 bits or more, 31 * 2^-14 of the sum of
    magnitudes at worst; over a whole result the rounding dominates, at most 2^-8 relative in the 2-norm.
  * experts, fp32: the error of p from its two products, carried through; where p lies nearer to a rounding boundary
    of its 8 bits than that, one step of its code either way; then the second product's.
  * experts, bfloat16: 2-norm, outputs' and partial rows' rounding (1.7e-3 each) and codes of p that the 8-bit
    instructions' error moves over a boundary (5e-4): 4e-3.
"""

import math
import sys

import numpy as np
import pytest

from tests import blocks_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch

    return torch


@pytest.fixture(scope="module")
def sd():
    import paper_1708_02937_amd as sd

    return sd


def _say(*a):
    print("[case]", *a, flush=True)


def _cuda(torch, a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _codes(torch, q):
    return q.view(torch.uint8).cpu().numpy()


def _to(torch, a, dtype):
    """float64 numpy rounded once to dtype's values (to nearest even), as float64."""
    if dtype == torch.float32:
        return a.astype(np.float32).astype(np.float64)
    return ref.round_bf16(a)


def _hidden(rng, shape, wide=True):
    x = rng.standard_normal(shape)
    if wide:
        x[..., rng.random(shape[-1]) < 0.02] *= 30
    return x


def _blocked(torch, sd, x, rows):
    """Operands from the reference's quantiser: (codes, scales) on the GPU and their float64 values."""
    flat = x.reshape(-1, *x.shape[-2:])
    both = [ref.quantize(m, rows) for m in flat]
    vals = np.stack([ref.values(c, s, x.shape[-1], rows) for c, s in both]).reshape(x.shape)
    codes = np.stack([c for c, _ in both]).reshape(*x.shape[:-1], -1)
    scales = np.stack([s for _, s in both])
    scales = scales.reshape(*x.shape[:-2], *scales.shape[1:])
    return _cuda(torch, codes).view(torch.float8_e4m3fn), _cuda(torch, scales).view(torch.float8_e8m0fnu), vals


# ------------------------------------------------------------------------------------------------ 8 bits


@pytest.mark.parametrize("rows,k,block_rows", [(1, 1, 1), (3, 127, 1), (5, 129, 128), (130, 300, 128), (257, 1000, 1),
                                               (128, 512, 128), (1, 4096, 128)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_blocks(torch, sd, rows, k, block_rows, dtype):
    rng = np.random.default_rng(rows * 1000 + k)
    x = _hidden(rng, (2, rows, k)) * 10.0 ** rng.integers(-6, 6, (2, rows, 1))
    x[rng.random(x.shape) < 0.05] = 0.0
    dt = getattr(torch, dtype)
    x = _to(torch, x, dt)
    _say("quantize", rows, k, block_rows, dtype)
    q, s = sd.quantize_blocks(_cuda(torch, x, dt), block_rows)
    for m in range(2):
        codes, scales = ref.quantize(x[m], block_rows)
        assert np.array_equal(_codes(torch, s[m]), scales)
        assert np.array_equal(_codes(torch, q[m]), codes)


def test_quantize_extremes(torch, sd):
    """Blocks of zeros, of subnormals, of the largest floats, at 448 and just above, with infinities and NaN."""
    x = np.zeros((9, 256), np.float32)
    x[1, :4] = [1e-45, -1e-40, 2.0 ** -127, 0]
    x[2, :3] = [3.4e38, -3.4e38, 1.0]
    x[3, :2] = [448, -1]
    x[4, :2] = [np.nextafter(np.float32(448), np.float32(1e9)), 1]
    x[5, :4] = [np.inf, 1, -2, 0.3]
    x[6, :4] = [np.nan, -np.inf, 5, 0.1]
    x[7, 128:132] = [np.inf, -np.inf, np.nan, 0]
    x[8, :] = -0.0
    q, s = sd.quantize_blocks(_cuda(torch, x))
    codes, scales = ref.quantize(x)
    got = _codes(torch, q)
    assert np.array_equal(_codes(torch, s), scales)
    nan = np.isnan(ref.TABLE[codes])
    assert np.array_equal(nan, (got & 127) == 127)
    assert np.array_equal(ref.TABLE[got][~nan], ref.TABLE[codes][~nan])


# ------------------------------------------------------------------------------------------------ norm


@pytest.mark.parametrize("rows,k", [(1, 1), (1, 4096), (3, 127), (5, 128), (7, 513), (2, 1025), (33, 2049), (9, 5000),
                                    (2, 16384), (3, 16385), (2, 32768), (777, 1001)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("res", [False, True])
def test_norm(torch, sd, rows, k, dtype, res):
    rng = np.random.default_rng(k + rows)
    dt = getattr(torch, dtype)
    x = _to(torch, _hidden(rng, (rows, k)), dt)
    r = _to(torch, _hidden(rng, (rows, k)), dt) if res else None
    g = (1 + 0.1 * rng.standard_normal(k)).astype(np.float32)
    _say("norm", rows, k, dtype, res)
    q, s, total, z = sd.norm_quantize(_cuda(torch, x, dt), _cuda(torch, g), 1e-6, normed=True,
                                      residual=None if r is None else _cuda(torch, r, dt))
    want_s, want_z = ref.norm(x, g, float(np.float32(1e-6)), r)
    codes, scales = ref.quantize(want_z)
    assert np.array_equal(_codes(torch, s), scales)
    assert np.array_equal(ref.TABLE[_codes(torch, q)], ref.TABLE[codes])
    assert np.array_equal(z.double().cpu().numpy(), _to(torch, want_z, dt))
    if res:  # the sum of two bfloat16 or float values is rounded to float, then to the type
        assert np.array_equal(total.double().cpu().numpy(), _to(torch, want_s.astype(np.float32), dt))
    else:
        assert total is None


def test_norm_rows_that_are_not_finite(torch, sd):
    """A row of zeros gives zeros (eps > 0); NaN spreads over its row; an infinity makes the rest of its row zero and
    itself NaN; other rows do not notice."""
    x = np.ones((6, 300), np.float32)
    x[1] = 0
    x[2, 5] = np.nan
    x[3, 7] = np.inf
    x[4] = 1e30  # squares overflow fp32
    x[5] = 1e-30
    q, s, _, z = sd.norm_quantize(_cuda(torch, x), torch.ones(300, device="cuda"), 1e-12, normed=True)
    z, v = z.cpu().numpy(), ref.TABLE[_codes(torch, q)][:, :300]
    assert np.array_equal(z[1], np.zeros(300)) and np.array_equal(v[1], np.zeros(300))
    assert np.isnan(z[2]).all() and np.isnan(v[2]).all()
    assert np.isnan(z[3, 7]) and np.isnan(v[3, 7]) and np.delete(z[3], 7).any() == 0
    assert np.allclose(z[0], 1) and np.allclose(z[4], 1)
    assert np.array_equal(_codes(torch, s)[2], np.ones(4))
    want = ref.norm(x[5:6], np.ones(300), float(np.float32(1e-12)))[1]
    assert np.array_equal(z[5], want[0].astype(np.float32))


def test_norm_strides_and_aliases(torch, sd):
    """Rows with strides, at odd addresses, and a sum written over the residual: the same results."""
    rng = np.random.default_rng(3)
    for dt in (torch.float32, torch.bfloat16):
        big = torch.randn(40, 700, device="cuda").to(dt)
        x, r = big[3:20, 5:506], big[21:38, 101:602]
        g = _cuda(torch, rng.standard_normal(501).astype(np.float32))
        a = sd.norm_quantize(x, g, residual=r, normed=True)
        b = sd.norm_quantize(x.contiguous(), g, residual=r.contiguous(), normed=True)
        for u, v in zip(a, b):
            assert torch.equal(u.view(torch.uint8) if u.element_size() == 1 else u,
                               v.view(torch.uint8) if v.element_size() == 1 else v)
        rest = r.clone()
        c = sd.norm_quantize(x, g, residual=rest, out_sum=rest)
        assert c[2] is rest and torch.equal(rest, a[2])
        assert torch.equal(c[0].view(torch.uint8), a[0].view(torch.uint8))


# ------------------------------------------------------------------------------------------------ routing

ROUTES = [
    # T, E, k, score, bias, groups, kept, best, normalize, factor
    (1, 1, 1, "softmax", False, 1, 1, 1, True, 1.0),
    (1, 64, 4, "softmax", False, 1, 1, 1, True, 1.0),
    (5, 7, 7, "sigmoid", True, 1, 1, 1, False, 2.5),
    (130, 60, 5, "sigmoid", True, 1, 1, 1, True, 1.0),
    (67, 65, 2, "softmax", True, 5, 2, 2, True, 1.0),
    (333, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5),
    (40, 128, 6, "softmax", False, 8, 3, 1, False, 1.0),
    (9, 1000, 64, "softmax", False, 1, 1, 1, True, 1.0),
    (3, 1024, 3, "sigmoid", False, 64, 1, 2, True, 1.0),
    (17, 64, 8, "sigmoid", True, 64, 8, 2, True, 1.0),
    (1025, 16, 2, "softmax", False, 4, 2, 1, True, 1.0),
    (4097, 33, 3, "softmax", False, 1, 1, 1, True, 1.0),
]


def _check_route(torch, sd, logits, dt, k, score, bias, groups, kept, best, normalize, factor):
    got = sd.route(_cuda(torch, logits, dt), k, score=score, bias=None if bias is None else _cuda(torch, bias),
                   groups=groups, groups_kept=kept, group_best=best, normalize=normalize, factor=factor)
    ids, weight = ref.route(logits, k, score, bias, groups, kept, best, normalize, factor)
    offsets, order = ref.plan(ids, logits.shape[1])
    assert np.array_equal(got.ids.cpu().numpy(), ids)
    assert np.all(np.abs(got.weight.cpu().numpy() - weight) <= 2.0 ** -23 * np.abs(weight) + 1e-45)
    assert np.array_equal(got.offsets.cpu().numpy(), offsets)
    assert np.array_equal(got.order.cpu().numpy(), order)


@pytest.mark.parametrize("T,E,k,score,use_bias,groups,kept,best,normalize,factor", ROUTES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_route(torch, sd, T, E, k, score, use_bias, groups, kept, best, normalize, factor, dtype):
    rng = np.random.default_rng(T + E)
    dt = getattr(torch, dtype)
    logits = _to(torch, 1.5 * rng.standard_normal((T, E)), dt)
    if T > 4:
        logits[rng.random(T) < 0.1] = -np.inf  # rows masked whole
        logits[rng.random((T, E)) < 0.05] = -np.inf  # experts masked for a token
        logits[rng.random((T, E)) < 0.01] = np.nan
    bias = (rng.integers(-100, 101, E) * np.float32(1e-3)).astype(np.float32) if use_bias else None
    _say("route", T, E, k, score, groups, dtype)
    _check_route(torch, sd, logits, dt, k, score, bias, groups, kept, best, normalize, factor)


def test_route_ties_and_extremes(torch, sd):
    """Equal logits go to the lower expert; rows with fewer live experts than places; infinite logits; logits so far
    apart that scores vanish; the lowest finite value as a mask."""
    for score in ("softmax", "sigmoid"):
        l = np.zeros((8, 70))
        l[1, 3:5] = 2.0
        l[2, :] = -np.inf
        l[2, 69] = 1.0
        l[3, 60] = np.inf
        l[4, [5, 50]] = np.inf
        l[5, :] = -3.3895313892515355e38
        l[5, 7] = 4.0
        l[6, :] = np.arange(70) * 20.0
        l[7, ::2] = np.nan
        for groups, kept, best in ((1, 1, 1), (7, 2, 2), (35, 3, 1)):
            with np.errstate(over="ignore"):
                _check_route(torch, sd, l, torch.float32, 6, score, None, groups, kept, best, True, 1.0)


def test_route_near_ties(torch, sd):
    """Logits one float apart, where 32-bit scores would be equal: the larger one wins all the same."""
    rng = np.random.default_rng(5)
    base = rng.standard_normal((64, 1)).astype(np.float32)
    l = np.repeat(base, 96, axis=1)
    for i in range(64):
        up = rng.permutation(96)[:5]
        for step, e in enumerate(up):
            for _ in range(step + 1):
                l[i, e] = np.nextafter(l[i, e], np.float32(np.inf))
    bias = np.zeros(96, np.float32)
    for score in ("softmax", "sigmoid"):
        _check_route(torch, sd, l.astype(np.float64), torch.float32, 4, score, bias, 1, 1, 1, True, 1.0)
        _check_route(torch, sd, l.astype(np.float64), torch.float32, 4, score, bias, 8, 3, 2, True, 1.0)


@pytest.mark.parametrize("T", [5, 40])
@pytest.mark.parametrize("E", [24, 70, 200, 300, 600])
def test_route_without_bias_by_logits(torch, sd, E, T):
    """Without a bias: logits one float apart, and different logits whose scores are the same in 64 bits too (a sigmoid
    of 1, scores of 0), which are ties."""
    rng = np.random.default_rng(E + T)
    l = np.repeat(rng.standard_normal((T, 1)).astype(np.float32), E, axis=1)
    for t in range(T):
        for step, e in enumerate(rng.permutation(E)[:5]):
            for _ in range(step + 1):
                l[t, e] = np.nextafter(l[t, e], np.float32(np.inf))
    l[1] = 45 + rng.permutation(E)  # sigmoids of 1
    l[2] = -2000 - rng.permutation(E)  # sigmoids of 0
    l[3] = -5000 - rng.permutation(E)  # softmax: 0 next to the first two
    l[3, [E - 1, E // 2]] = [1.0, 0.5]
    for score in ("softmax", "sigmoid"):
        for groups, kept, best in ((1, 1, 1), (2, 1, 2)):
            _say("route by logits", T, E, score, groups)
            with np.errstate(over="ignore"):
                _check_route(torch, sd, l.astype(np.float64), torch.float32, 4, score, None, groups, kept, best, True, 1.0)


@pytest.mark.parametrize("T,E,k,score,use_bias,groups,kept,best", [
    (8, 300, 8, "sigmoid", True, 4, 2, 2), (100, 300, 8, "sigmoid", True, 4, 2, 2), (100, 512, 8, "softmax", True, 8, 4, 2),
    (33, 1000, 5, "softmax", False, 8, 3, 2), (70, 1024, 8, "sigmoid", True, 8, 4, 2), (19, 513, 17, "softmax", False, 1, 1, 1),
])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_route_many_experts(torch, sd, T, E, k, score, use_bias, groups, kept, best, dtype):
    rng = np.random.default_rng(T * E)
    dt = getattr(torch, dtype)
    logits = _to(torch, 1.5 * rng.standard_normal((T, E)), dt)
    logits[rng.random((T, E)) < 0.1] = -np.inf
    bias = (rng.integers(-100, 101, E) * np.float32(1e-3)).astype(np.float32) if use_bias else None
    _say("route", T, E, k, score, groups, dtype)
    _check_route(torch, sd, logits, dt, k, score, bias, groups, kept, best, True, 2.5)


def test_route_strides_and_empty(torch, sd):
    big = torch.randn(50, 90, device="cuda")
    a, b = sd.route(big[3:40, 7:67], 3), sd.route(big[3:40, 7:67].contiguous(), 3)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    r = sd.route(torch.empty(0, 12, device="cuda"), 2)
    assert r.ids.shape == (0, 2) and r.offsets.tolist() == [0] * 13 and r.order.numel() == 0


# ------------------------------------------------------------------------------------------------ product

PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 4096, 4096), (2, 100, 130), (16, 64, 256), (17, 129, 1001), (33, 300, 640),
            (63, 257, 384), (64, 128, 128), (65, 260, 511), (128, 256, 1024), (129, 1000, 2001), (255, 513, 900),
            (300, 700, 4000), (777, 299, 1001), (1024, 512, 640)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_product(torch, sd, m, n, k, dtype):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    dt = getattr(torch, dtype)
    a, sa, av = _blocked(torch, sd, _hidden(rng, (m, k)), 1)
    w, sw, wv = _blocked(torch, sd, rng.standard_normal((n, k)) / math.sqrt(k) * 4.0 ** rng.integers(-3, 3, (n, 1)),
                         128)
    bias = (0.1 * rng.standard_normal(n)).astype(np.float32)
    y, big = av @ wv.T, np.abs(av) @ np.abs(wv).T
    for use_bias, ymax in ((False, None), (True, math.inf), (True, 0.5)):
        _say("product", m, n, k, dtype, use_bias, ymax)
        got = sd.product_blocks(a, sa, w, sw, k, bias=_cuda(torch, bias) if use_bias else None, ymax=ymax, dtype=dt)
        got = got.double().cpu().numpy()
        z, S = (y + bias, big + np.abs(bias)) if use_bias else (y, big)
        want = z if ymax is None else np.clip(z, 0, ymax)
        if dt == torch.float32:
            assert np.all(np.abs(got - want) <= (k + 16) * 2.0 ** -24 * S)
        else:
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 31 * 2.0 ** -14 * S)
            assert np.linalg.norm(got - want) <= 2.0 ** -8 * np.linalg.norm(want)


def test_product_of_integers_is_exact(torch, sd):
    """Small integers: every product and sum is exact in both arithmetics, whatever the tile a row falls into."""
    rng = np.random.default_rng(1)
    for m, n, k in ((5, 40, 300), (70, 300, 1000), (300, 520, 700), (4100, 4097, 200)):
        a, sa, av = _blocked(torch, sd, rng.integers(-4, 5, (m, k)).astype(float), 1)
        w, sw, wv = _blocked(torch, sd, rng.integers(-4, 5, (n, k)).astype(float), 128)
        for dt in (torch.float32, torch.bfloat16):
            got = sd.product_blocks(a, sa, w, sw, k, dtype=dt).double().cpu().numpy()
            assert np.array_equal(got, _to(torch, av @ wv.T, dt)), (m, n, k, dt)


@pytest.mark.parametrize("m,n,k", [(20, 70, 33000), (3, 8200, 300), (16, 40, 70000), (300, 200, 31900), (70, 300, 65600)])
def test_product_long_rows(torch, sd, m, n, k):
    """Rows whose scales do not all fit in LDS, and the few-row kernel on both sides of its width: exact integers."""
    rng = np.random.default_rng(m)
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randint(-2, 3, (m, k), generator=g, device="cuda").float()
    y = torch.randint(-2, 3, (n, k), generator=g, device="cuda").float()
    a, sa = sd.quantize_blocks(x)
    w, sw = sd.quantize_blocks(y, 128)
    want = (x.double() @ y.double().t()).cpu().numpy()
    for dt in (torch.float32, torch.bfloat16):
        _say("long rows", m, n, k, dt)
        got = sd.product_blocks(a, sa, w, sw, k, dtype=dt).double().cpu().numpy()
        assert np.array_equal(got, _to(torch, want, dt))


@pytest.mark.parametrize("m,n,k", [(33, 1000, 3999), (116, 271, 1287), (250, 250, 640), (8, 8192, 130), (9, 4097, 257),
                                   (64, 4200, 1001), (257, 1000, 4000), (500, 900, 333), (1000, 2000, 2500),
                                   (400, 700, 33000), (600, 260, 66000)])
def test_product_between_few_rows_and_tiles(torch, sd, m, n, k):
    """Both sides of the bound between 16 x 16 outputs per workgroup and larger tiles, rows too long for their scales to
    lie in LDS among these: exact integers."""
    g = torch.Generator(device="cuda").manual_seed(m + n)
    x = torch.randint(-2, 3, (m, k), generator=g, device="cuda").float()
    y = torch.randint(-2, 3, (n, k), generator=g, device="cuda").float()
    a, sa = sd.quantize_blocks(x)
    w, sw = sd.quantize_blocks(y, 128)
    bias = torch.randint(-9, 10, (n,), generator=g, device="cuda").float()
    want = (x.double() @ y.double().t()).cpu().numpy() + bias.double().cpu().numpy()
    for dt in (torch.float32, torch.bfloat16):
        _say("few rows or tiles", m, n, k, dt)
        got = sd.product_blocks(a, sa, w, sw, k, bias=bias, ymax=150.0, dtype=dt).double().cpu().numpy()
        assert np.array_equal(got, _to(torch, np.clip(want, 0, 150.0), dt))


def test_product_extremes(torch, sd):
    """Scales at both ends of their range, NaN codes in one row and one column only, outputs in a strided view."""
    m, n, k = 40, 150, 300
    rng = np.random.default_rng(2)
    a, sa, _ = _blocked(torch, sd, rng.standard_normal((m, k)), 1)
    w, sw, _ = _blocked(torch, sd, rng.standard_normal((n, k)), 128)
    sa.view(torch.uint8)[3] = 1
    sa.view(torch.uint8)[4] = 200
    sw.view(torch.uint8)[1] = 60
    a.view(torch.uint8)[7, 5] = 0x7F
    w.view(torch.uint8)[9, 299] = 0xFF
    av = ref.values(_codes(torch, a), _codes(torch, sa), k)
    wv = ref.values(_codes(torch, w), _codes(torch, sw), k, 128)
    want = av @ wv.T
    nan = np.isnan(want)
    assert nan[7].all() and nan[:, 9].all() and nan.sum() == m + n - 1
    S = np.abs(np.nan_to_num(av)) @ np.abs(np.nan_to_num(wv)).T
    for dt in (torch.float32, torch.bfloat16):
        y = torch.full((m, n + 13), 7.0, device="cuda", dtype=dt)
        sd.product_blocks(a, sa, w, sw, k, dtype=dt, out=y[:, 5:5 + n])
        got = y.double().cpu().numpy()
        assert np.all(got[:, :5] == 7) and np.all(got[:, 5 + n:] == 7)
        got = got[:, 5:5 + n]
        assert np.array_equal(np.isnan(got), nan)
        tol = (k + 16) * 2.0 ** -24 * S if dt == torch.float32 else 2.0 ** -8 * np.abs(want) + 31 * 2.0 ** -14 * S
        assert np.all(np.abs(got - want)[~nan] <= tol[~nan] + 1e-37)


# ------------------------------------------------------------------------------------------------ experts

EXPERTS = [
    # T, H, F, E, k, masked share
    (1, 256, 128, 4, 2, 0.0),
    (1, 300, 70, 8, 8, 0.0),
    (3, 129, 257, 5, 1, 0.0),
    (20, 500, 300, 6, 3, 0.2),
    (65, 640, 200, 4, 2, 0.1),
    (300, 257, 130, 3, 2, 0.1),
    (700, 256, 384, 2, 1, 0.0),
    (64, 128, 128, 40, 4, 0.5),
    (5, 200, 100, 64, 2, 1.0),
]


def _experts_case(torch, sd, T, H, F, E, k, masked, seed=0):
    rng = np.random.default_rng(T + H + F + seed)
    a, sa, av = _blocked(torch, sd, _hidden(rng, (T, H)), 1)
    w1, s1, v1 = _blocked(torch, sd, rng.standard_normal((E, 2, F, H)) / math.sqrt(H), 128)
    w2, s2, v2 = _blocked(torch, sd, rng.standard_normal((E, H, F)) / math.sqrt(F), 128)
    logits = 1.5 * rng.standard_normal((T, E)) + rng.standard_normal(E)
    logits[rng.random(T) < masked] = -np.inf
    ids, weight = ref.route(logits, k, "softmax", None, 1, 1, 1, True, 1.0)
    ids[rng.random((T, k)) < masked / 4] = -1  # places without an expert beside ones with
    weight = np.where(ids < 0, 0, weight).astype(np.float32)
    offsets, order = ref.plan(ids, E)
    routes = sd.Routes(*(_cuda(torch, x) for x in (ids, weight, offsets, order)))
    residual = rng.standard_normal((T, H))
    return (a, sa, routes, w1, s1, w2, s2), (av, v1, v2, ids, weight), residual


def _experts_ref(av, v1, v2, ids, weight, exact):
    """(out, bound on the error of an fp32 run) by the definition, slot by slot."""
    T, H = av.shape
    E, _, F, _ = v1.shape
    out, tol = np.zeros((T, H)), np.zeros((T, H))
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if t.size == 0:
            continue
        x = av[t]
        g, u = x @ v1[e, 0].T, x @ v1[e, 1].T
        sig = 1 / (1 + np.exp(-g))
        p = g * sig * u
        codes, scales = ref.quantize(p)
        q = ref.values(codes, scales, F)
        o = q @ v2[e].T
        wt = weight[t, j].astype(np.float64)[:, None]
        np.add.at(out, t, wt * o)
        if exact:
            u24 = 2.0 ** -24
            eg, eu = ((H + 16) * u24 * (np.abs(x) @ np.abs(v1[e, i]).T) for i in (0, 1))
            dp = 1.1 * np.abs(u) * eg + np.abs(g * sig) * eu + 16 * u24 * np.abs(p)
            # a scale may move where the block's largest value is that near to a boundary: no test value is
            unit = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 128, axis=1)[:, :F]
            step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(p) / unit, 2.0 ** -6))) - 3), 2.0 ** -9) * unit
            edge = np.abs(np.abs(p - q) - step / 2)  # distance to the nearest rounding boundary
            move = np.where(edge <= dp + 1e-12 * unit, step, 0.0)
            d = move @ np.abs(v2[e]).T + (F + 32) * u24 * (np.abs(q) @ np.abs(v2[e]).T)
            np.add.at(tol, t, np.abs(wt) * d)
    return out, tol


@pytest.mark.parametrize("T,H,F,E,k,masked", EXPERTS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("res", [False, True])
def test_experts(torch, sd, T, H, F, E, k, masked, dtype, res):
    dt = getattr(torch, dtype)
    args, host, residual = _experts_case(torch, sd, T, H, F, E, k, masked)
    want, tol = _experts_ref(*host, dt == torch.float32)
    r = None
    if res:
        residual = _to(torch, residual, dt)
        want = want + residual
        r = _cuda(torch, residual, dt)
    _say("experts", T, H, F, E, k, dtype, res)
    got = sd.experts_forward(*args, H, F, residual=r, dtype=dt).double().cpu().numpy()
    if dt == torch.float32:
        assert np.all(np.abs(got - want) <= tol + (k + 4) * 2.0 ** -24 * (np.abs(want) + tol + np.abs(residual) * res)
                      + 1e-6 * tol)
    elif np.linalg.norm(want) > 0:
        assert np.linalg.norm(got - want) <= 4e-3 * np.linalg.norm(want)
    dead = (host[3] < 0).all(axis=1)
    assert np.array_equal(got[dead], residual[dead] if res else np.zeros((dead.sum(), H)))


@pytest.mark.parametrize("T,H,F,E,k", [(64, 129, 33000, 2, 2), (70, 80000, 130, 2, 1), (2, 33000, 70, 4, 2),
                                       (1500, 260, 900, 8, 2)])
def test_experts_of_any_shape(torch, sd, T, H, F, E, k):
    """Long inner and outer rows, and enough tiles for the largest kind, against float64 on the GPU (2-norm, as above)."""
    g = torch.Generator(device="cuda").manual_seed(T)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    a, sa = sd.quantize_blocks(rand(T, H))
    w1, s1 = sd.quantize_blocks(rand(E, 2, F, H) / H ** 0.5, 128)
    w2, s2 = sd.quantize_blocks(rand(E, H, F) / F ** 0.5, 128)
    routes = sd.route(rand(T, E), k)
    _say("experts", T, H, F, E, k)
    got = sd.experts_forward(a, sa, routes, w1, s1, w2, s2, H, F).double()

    def value(c, s, rows, n, m):
        e = torch.exp2(s.view(torch.uint8).double() - 127).repeat_interleave(rows, 0)[:n]
        return (c.double().unflatten(1, (-1, 128)) * e[:, :c.shape[1] // 128, None]).flatten(1)[:, :m]

    x, want = value(a, sa, 1, T, H), torch.zeros(T, H, dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = (routes.ids == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        gate, up = (x[t] @ value(w1[e, i], s1[e, i], 128, F, H).t() for i in (0, 1))
        p = (gate * torch.sigmoid(gate) * up).cpu().numpy()
        q = torch.from_numpy(ref.values(*ref.quantize(p), F)).cuda()
        want.index_add_(0, t, (q @ value(w2[e], s2[e], 128, H, F).t()) * routes.weight[t, j].double()[:, None])
    assert float((got - want).norm() / want.norm()) <= 4e-3


def test_experts_rows_that_are_not_finite(torch, sd):
    """A NaN code in one token's row, and weights so large that one expert's products overflow: the token and the
    expert's tokens are lost, the others do not notice."""
    for T in (2, 200):
        H, F, E = 256, 256, 4
        args, host, _ = _experts_case(torch, sd, T, H, F, E, 1, 0.0, seed=7)
        for dt in (torch.float32, torch.bfloat16):
            want = sd.experts_forward(*args, H, F, dtype=dt)
            a = args[0].clone()
            a.view(torch.uint8)[1, 3] = 0x7F
            got = sd.experts_forward(a, *args[1:], H, F, dtype=dt)
            rest = torch.arange(T, device="cuda") != 1
            assert torch.isnan(got[1]).all() and torch.equal(got[rest], want[rest])
            s_out = args[6].clone()
            hit = int(host[3][0, 0])
            s_out.view(torch.uint8)[hit, 1] = 254  # outputs 128 on of that expert: 2^127 times the codes
            got = sd.experts_forward(*args[:6], s_out, H, F, dtype=dt)
            other = (args[2].ids != hit).all(dim=1)
            assert torch.equal(got[other], want[other])
            assert torch.equal(got[:, :128], want[:, :128])
            assert not torch.isfinite(got[~other][:, 128:]).all()


def test_experts_in_place_and_workspace(torch, sd):
    """The output over the residual, a strided output, and a workspace of the caller's full of NaN: same results."""
    T, H, F, E, k = 33, 260, 140, 5, 2
    args, _, residual = _experts_case(torch, sd, T, H, F, E, k, 0.1)
    r = _cuda(torch, residual, torch.bfloat16)
    want = sd.experts_forward(*args, H, F, residual=r)
    need = sd.sdnn_experts_workspace_size(T, H, F, E, k, sd.SDNN_TYPE_BF16)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    over = r.clone()
    assert torch.equal(sd.experts_forward(*args, H, F, residual=over, out=over, ws=ws), want)
    wide = torch.zeros(T, H + 9, dtype=torch.bfloat16, device="cuda")
    sd.experts_forward(*args, H, F, residual=r, out=wide[:, 3:3 + H], ws=ws)
    assert torch.equal(wide[:, 3:3 + H], want) and not wide[:, :3].any() and not wide[:, 3 + H:].any()


# ------------------------------------------------------------------------------------------------ together


def _layer(sd, torch, x, r, gamma, w_router, weights, k, H, F):
    q, s, total, z = sd.norm_quantize(x, gamma, residual=r, normed=True)
    routes = sd.route((z.float() @ w_router).contiguous(), k)
    return sd.experts_forward(q, s, routes, *weights, H, F, residual=total, dtype=x.dtype)


@pytest.mark.parametrize("T", [1, 200])
def test_layer_on_a_side_stream_and_in_a_graph(torch, sd, T):
    """The whole layer on another stream than the default one, and captured: every replay equals the eager result on
    that replay's inputs, with eager work and synchronisations in between."""
    H, F, E, k = 384, 256, 8, 2
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    weights = (*sd.quantize_blocks(rand(E, 2, F, H) / H ** 0.5, 128), *sd.quantize_blocks(rand(E, H, F) / F ** 0.5, 128))
    gamma, w_router = torch.ones(H, device="cuda"), rand(H, E) / H ** 0.5
    x, r = rand(T, H).bfloat16(), rand(T, H).bfloat16()
    want = _layer(sd, torch, x, r, gamma, w_router, weights, k, H, F)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2 = (x.float() * 2).bfloat16()  # made on the side stream just before
        got = _layer(sd, torch, (x2.float() / 2).bfloat16(), r, gamma, w_router, weights, k, H, F)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(sd, torch, x, r, gamma, w_router, weights, k, H, F)
    for i in range(4):
        x.copy_(rand(T, H).bfloat16())
        want = _layer(sd, torch, x, r, gamma, w_router, weights, k, H, F)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_example(torch, sd, capsys):
    """The example's prompt and its captured single token: the token's row is the prompt's.  Each of the two layers rounds
    its input to 8 bits, where a difference of one bfloat16 rounding (2^-9) moves about one code in twenty by a step of a
    sixteenth to an eighth: 1 to 2% of a layer's result."""
    import examples.experts_layer as example

    far = example.main(["--width", "512", "--inner", "256", "--experts", "8", "--chosen", "2", "--prompt", "200"])
    assert far <= 0.05
    assert "tokens/s" in capsys.readouterr().out


def test_same_inputs_same_bits(torch, sd):
    T, H, F, E, k = 130, 512, 256, 6, 3
    args, _, _ = _experts_case(torch, sd, T, H, F, E, k, 0.0)
    a = sd.experts_forward(*args, H, F)
    for _ in range(3):
        assert torch.equal(sd.experts_forward(*args, H, F), a)


# ------------------------------------------------------------------------------------------------ tensor arguments


def test_tensor_arguments_are_checked(torch, sd):
    """Wrong types, shapes, devices and strides are ValueErrors (TypeError where no tensor is given); what only the C call
    refuses carries its status."""
    x = torch.randn(6, 200, device="cuda")
    gamma = torch.ones(200, device="cuda")
    a, sa = sd.quantize_blocks(x)
    w, sw = sd.quantize_blocks(torch.randn(70, 200, device="cuda"), 128)
    logits = torch.randn(6, 8, device="cuda")
    routes = sd.route(logits, 2)
    w_in, s_in = sd.quantize_blocks(torch.randn(8, 2, 40, 200, device="cuda"), 128)
    w_out, s_out = sd.quantize_blocks(torch.randn(8, 200, 40, device="cuda"), 128)

    def experts(**kw):
        args = dict(a=a, a_scale=sa, routes=routes, w_in=w_in, w_in_scale=s_in, w_out=w_out, w_out_scale=s_out, width=200,
                    inner=40)
        return sd.experts_forward(**{**args, **kw})

    assert experts().shape == (6, 200)
    wrong = [
        lambda: sd.norm_quantize(x.half(), gamma), lambda: sd.norm_quantize(x[0], gamma),
        lambda: sd.norm_quantize(x, gamma[1:]), lambda: sd.norm_quantize(x, gamma.double()),
        lambda: sd.norm_quantize(x, gamma.cpu()), lambda: sd.norm_quantize(x.t(), torch.ones(6, device="cuda")),
        lambda: sd.norm_quantize(x, gamma, residual=x.bfloat16()), lambda: sd.norm_quantize(x, gamma, residual=x[1:]),
        lambda: sd.norm_quantize(x, gamma, out_sum=x), lambda: sd.quantize_blocks(x.t()),
        lambda: sd.quantize_blocks(x[0]), lambda: sd.product_blocks(a, sa, w, sw, 300),
        lambda: sd.product_blocks(a[:5], sa, w, sw, 200), lambda: sd.product_blocks(a, sa, w, sw[:, :2], 200),
        lambda: sd.product_blocks(a.view(torch.uint8), sa, w, sw, 200),
        lambda: sd.product_blocks(a, sa, w, sw, 200, bias=gamma), lambda: sd.product_blocks(a, sa, w, sw, 200, out=x),
        lambda: sd.product_blocks(a, sa, w, sw, 200, dtype=torch.float16), lambda: sd.route(logits, 0),
        lambda: sd.route(logits, 2, score="best"), lambda: sd.route(logits.long(), 2),
        lambda: sd.route(logits, 2, bias=gamma), lambda: experts(a=a[:3]), lambda: experts(w_out=w_out[:4]),
        lambda: experts(residual=x), lambda: experts(ws=torch.empty(9, device="cuda")), lambda: experts(width=201),
        lambda: experts(routes=routes._replace(order=routes.order[1:])),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"case {i} was taken")
    for call in (lambda: sd.norm_quantize(x, None), lambda: sd.route(logits, 2.5), lambda: sd.route(logits, 2, bias=3)):
        with pytest.raises(TypeError):
            call()
    for status, call in ((2, lambda: sd.route(logits, 9)), (2, lambda: sd.norm_quantize(x, gamma, eps=-1.0)),
                         (2, lambda: sd.quantize_blocks(x, 64)), (2, lambda: sd.route(logits, 2, groups=3)),
                         (6, lambda: experts(ws=torch.empty(16, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(sd.SdnnError) as e:
            call()
        assert e.value.status == status


def test_tensor_results_are_owned(torch, sd):
    """Results are freed when they are dropped, out tensors come back as themselves, refused calls keep nothing."""
    x = torch.randn(64, 500, device="cuda")
    gamma = torch.ones(500, device="cuda")
    same = sd.norm_quantize(x, gamma, residual=x.clone(), out_sum=x)
    assert same[2] is x and same[3] is None
    del same
    torch.cuda.synchronize()
    before, refs = torch.cuda.memory_allocated(), sys.getrefcount(x)
    for _ in range(20):
        sd.norm_quantize(x, gamma, residual=x, normed=True)
        sd.route(x, 3)
        sd.product_blocks(*sd.quantize_blocks(x), *sd.quantize_blocks(x, 128), 500)
        with pytest.raises(sd.SdnnError):
            sd.route(x, 501)
    assert torch.cuda.memory_allocated() == before and sys.getrefcount(x) == refs
