"""Every kind of tile that the products of blocked 8-bit matrices are computed on, over enough blocks that its ring of
stages turns around and its scales are sent for more than once, with scales that differ by row, block and block row.

Which kind a size takes is written down here a second time (kind_of, experts_kind): a change of the rule has to change
the sizes below too, so that every kind stays covered.

Tolerances, fixed before any run:
  * products of small integers times powers of two: equal.  Every product and partial sum is a multiple of 2^-4 below
    2^18 (|x|, |w| <= 8, 128 products of a block, 21 blocks), which fp32 holds, and the products of one instruction have
    one scale, so that none is dropped; one rounding to bfloat16.
  * extremes: K products summed in fp32 in any order, (K + 16) 2^-24 of the sum of magnitudes; with the 8-bit
    instructions 31 * 2^-14 of it at worst and the output's rounding.  Where that sum passes the largest float nothing
    is asked.
  * accuracy of bfloat16 products of normal values: what the 8-bit instructions drop, 1.5e-5, beside the output's rounding,
    1.7e-3, both as 2-norms and independent: 1.0001 times the rounding alone, and 1.01 for chance.
  * experts, bfloat16, first product exact: rows held at 11 bits until they are summed, 1.4e-4, and the second product's
    1.5e-5, beside the rounding: 1.004 times it, and 1.03 for chance.  With both products on the 8-bit instructions some
    codes of p move over a boundary: 1.17 to 1.55 times the rounding without a residual over many calls, 1.03 to 1.31 with
    one; 1.7 and 1.45.
  * experts, float: p is about 1e-6 off, which moves about 3e-5 of its codes by a step of 0.09: 5e-4 in the 2-norm; 1e-3.
"""

import math

import pytest

gpu = pytest.mark.gpu
BF16, F32 = "bfloat16", "float32"


def up(a, b):
    return -(-a // b)


def kind_of(m, n, k, dtype):
    """The kernel of a product: 'few', or (outputs, rows, groups of waves) of a tile."""
    cells = up(m, 16) * up(n, 16)
    if cells <= (256 if dtype == BF16 and m > 8 else 512):
        return "few"
    small, words = up(m, 64) * up(n, 64), up(up(k, 128), 4) * 4 + 4
    room = 160 * 1024
    if small <= 1024 and 4 * 256 * 64 * 2 + 129 * words <= room and 3 * 192 * 64 * 4 + 65 * words <= room:
        if small <= (128 if dtype == BF16 else 256):
            return 64, 64, 4
        if dtype == BF16 and small <= 256:
            return 64, 64, 2
        if small <= 512:
            return 128, 64, 2 if dtype == BF16 else 4
        return (64, 64, 1) if k <= 2048 else (128, 128, 2)
    if dtype == F32:
        return 128, 128, 1
    return (256, 128, 1) if small <= 2048 else (256, 256, 1)


def experts_kind(T, width, inner, E, k, dtype):
    """'few', or (rows of a tile, groups of waves of the first product)."""
    slots = T * k
    if slots <= E:
        return "few"
    busy = min(slots, E)
    if dtype == BF16 and slots >= 32 * busy and (busy + slots // 128) * up(inner, 128) >= 400:
        return 128, 1
    return 64, 2 if 3 * 320 * 64 * 2 + 66 * (up(up(width, 128), 4) * 4 + 4) <= 160 * 1024 else 1


KINDS = [
    (BF16, "few", 60, 1000, 2561), (BF16, (64, 64, 4), 100, 1000, 2561), (BF16, (64, 64, 2), 200, 4000, 2561),
    (BF16, (128, 64, 2), 400, 4100, 2561), (BF16, (64, 64, 1), 777, 2999, 1951),
    (BF16, (128, 128, 2), 777, 2999, 2561), (BF16, (256, 128, 1), 1000, 5000, 2561),
    (BF16, (256, 128, 1), 100, 1000, 33001), (BF16, (256, 256, 1), 1500, 6001, 2561),
    (BF16, (256, 256, 1), 4097, 2310, 1409), (F32, "few", 100, 1000, 2561), (F32, (64, 64, 4), 200, 3999, 2561),
    (F32, (128, 64, 4), 400, 4100, 2561), (F32, (64, 64, 1), 777, 2999, 1951), (F32, (128, 128, 2), 777, 2999, 2561),
    (F32, (128, 128, 1), 1000, 5000, 2561), (F32, (128, 128, 1), 200, 1000, 33001),
]
EXPERTS = [
    # dtype, kind, T, H, F, E, k, masked share, residual
    (BF16, (128, 1), 3000, 700, 900, 8, 2, 0.0, False),
    (BF16, (128, 1), 3000, 2601, 900, 8, 2, 0.1, True),
    (BF16, (128, 1), 5000, 520, 2600, 5, 1, 0.0, True),
    (BF16, (64, 2), 500, 2601, 700, 6, 3, 0.1, False),
    (BF16, (64, 2), 333, 520, 2600, 6, 2, 0.0, True),
    (F32, (64, 2), 500, 2601, 700, 6, 3, 0.1, True),
    (F32, (64, 2), 3000, 700, 900, 8, 2, 0.0, False),
    (F32, (64, 1), 200, 80000, 150, 3, 2, 0.0, False),
    (BF16, (64, 1), 200, 80000, 150, 3, 2, 0.0, False),
]


def test_every_kind_is_reached():
    for dtype, kind, m, n, k in KINDS:
        assert kind_of(m, n, k, dtype) == kind, (dtype, m, n, k)
    assert {kind for d, kind, *_ in KINDS if d == BF16} == {
        "few", (64, 64, 4), (64, 64, 2), (128, 64, 2), (64, 64, 1), (128, 128, 2), (256, 128, 1), (256, 256, 1)}
    assert {kind for d, kind, *_ in KINDS if d == F32} == {
        "few", (64, 64, 4), (128, 64, 4), (64, 64, 1), (128, 128, 2), (128, 128, 1)}
    for dtype, kind, T, H, F, E, k, _, _ in EXPERTS:
        assert experts_kind(T, H, F, E, k, dtype) == kind, (dtype, T, H, F, E, k)


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


def _values(torch, codes, scales, block_rows, k):
    """float64 values of a blocked matrix."""
    s = torch.exp2(scales.view(torch.uint8).double() - 127).repeat_interleave(block_rows, 0)[:codes.shape[0]]
    v = codes.double().unflatten(1, (-1, 128)) * s[:, :codes.shape[1] // 128, None]
    return v.flatten(1)[:, :k]


def _integers(torch, g, rows, k, block_rows):
    """Integers up to 2 times a power of two from 1/4 to 4 for each block: exact in 8 bits, with scales all over."""
    x = torch.randint(-2, 3, (rows, k), generator=g, device="cuda").double()
    e = torch.randint(-2, 3, (up(rows, block_rows), up(k, 128)), generator=g, device="cuda").double()
    return x * torch.exp2(e).repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :k]


@gpu
@pytest.mark.parametrize("dtype,kind,m,n,k", KINDS)
def test_scales_that_differ(torch, sd, dtype, kind, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    dt = getattr(torch, dtype)
    x, y = _integers(torch, g, m, k, 1), _integers(torch, g, n, k, 128)
    if k > 4096:  # partial sums as small as above: one block in sixteen is not zero
        x *= (torch.arange(k, device="cuda") // 128 % 16 == 3)
    a, sa = sd.quantize_blocks(x.float())
    w, sw = sd.quantize_blocks(y.float(), 128)
    assert torch.equal(_values(torch, a, sa, 1, k), x) and torch.equal(_values(torch, w, sw, 128, k), y)
    bias = torch.randint(-9, 10, (n,), generator=g, device="cuda").float()
    want = x @ y.t()
    _say("scales that differ", dtype, kind, m, n, k)
    assert torch.equal(sd.product_blocks(a, sa, w, sw, k, dtype=dt), want.float().to(dt))
    want = (want + bias.double()).clamp(0, 150)
    got = sd.product_blocks(a, sa, w, sw, k, bias=bias, ymax=150.0, dtype=dt)
    assert torch.equal(got, want.float().to(dt))


@gpu
@pytest.mark.parametrize("dtype,kind,m,n,k", KINDS)
def test_extremes(torch, sd, dtype, kind, m, n, k):
    """Scales at both ends of their range, NaN codes in one row and one column, outputs in a view at an odd place."""
    g = torch.Generator(device="cuda").manual_seed(m * n + k)
    dt = getattr(torch, dtype)
    a, sa = sd.quantize_blocks(torch.randn(m, k, generator=g, device="cuda"))
    w, sw = sd.quantize_blocks(torch.randn(n, k, generator=g, device="cuda"), 128)
    spread = torch.randint(-6, 7, sw.shape, generator=g, device="cuda")
    sw = (sw.view(torch.uint8).int() + spread).to(torch.uint8).view(sw.dtype)
    sa.view(torch.uint8)[3] = 1
    sa.view(torch.uint8)[m - 4] = 200
    sa.view(torch.uint8)[4, ::2] = 250
    sw.view(torch.uint8)[1] = 60
    a.view(torch.uint8)[7, 5] = 0x7F
    w.view(torch.uint8)[9, k - 1] = 0xFF
    x, y = _values(torch, a, sa, 1, k), _values(torch, w, sw, 128, k)
    want, size = x @ y.t(), x.nan_to_num().abs() @ y.nan_to_num().abs().t()
    nan = want.isnan()
    assert bool(nan[7].all()) and bool(nan[:, 9].all()) and int(nan.sum()) == m + n - 1
    wide = torch.full((m, n + 13), 7.0, device="cuda", dtype=dt)
    _say("extremes", dtype, kind, m, n, k)
    sd.product_blocks(a, sa, w, sw, k, dtype=dt, out=wide[:, 5:5 + n])
    assert bool((wide[:, :5] == 7).all()) and bool((wide[:, 5 + n:] == 7).all())
    got = wide[:, 5:5 + n].double()
    fits = size < 3e38  # not so for row 4, but for the block row of small weights
    assert bool(fits[:4].all()) and bool(fits[5:].all()) and bool(fits[4, 128:256].all())
    assert torch.equal(got.isnan()[fits], nan[fits])
    dropped = 31 * 2.0 ** -14 * size + 2.0 ** -8 * want.abs()
    tolerance = ((k + 16) * 2.0 ** -24 * size if dtype == F32 else dropped) + 1e-37
    assert bool(((got - want).abs() <= tolerance)[~nan & fits].all())


@gpu
@pytest.mark.parametrize("dtype,kind,m,n,k", KINDS)
def test_accuracy(torch, sd, dtype, kind, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(m + 3 * n + k)
    dt = getattr(torch, dtype)
    a, sa = sd.quantize_blocks(torch.randn(m, k, generator=g, device="cuda"))
    w, sw = sd.quantize_blocks(torch.randn(n, k, generator=g, device="cuda") / k ** 0.5, 128)
    x, y = _values(torch, a, sa, 1, k), _values(torch, w, sw, 128, k)
    want = x @ y.t()
    _say("accuracy", dtype, kind, m, n, k)
    off = (sd.product_blocks(a, sa, w, sw, k, dtype=dt).double() - want).norm()
    if dtype == BF16:
        assert float(off) <= 1.01 * float((want.bfloat16().double() - want).norm())
    else:
        assert float(off) <= (k + 16) * 2.0 ** -24 * float((x.abs() @ y.abs().t()).norm())


def _rounded8(torch, p):
    """float64 rows after their rounding to 8 bits in blocks of 128, as float64 values."""
    rows, k = p.shape
    t = torch.nn.functional.pad(p, (0, up(k, 128) * 128 - k)).view(rows, -1, 128)
    m, e = torch.frexp(t.abs().amax(dim=2, keepdim=True))
    scale = torch.exp2((e - 9 + (m > 0.875).int()).clamp(min=-126).double())
    v = t / scale
    step = torch.exp2(torch.frexp(v)[1].clamp(min=-5).double() - 4)
    return (torch.round(v / step) * step * scale).view(rows, -1)[:, :k]


@gpu
@pytest.mark.parametrize("dtype,kind,T,H,F,E,k,masked,residual", EXPERTS)
def test_experts(torch, sd, dtype, kind, T, H, F, E, k, masked, residual):
    """Several tiles to an expert, full ones and cut ones, over several runs of outputs; uneven experts, one of them empty."""
    g = torch.Generator(device="cuda").manual_seed(T + H + F)
    dt = getattr(torch, dtype)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    a, sa = sd.quantize_blocks(rand(T, H))
    block = torch.exp2(torch.randint(-2, 3, (E, 2, 1, 1), generator=g, device="cuda").float())
    w1, s1 = sd.quantize_blocks(rand(E, 2, F, H) / H ** 0.5 * block, 128)
    w2, s2 = sd.quantize_blocks(rand(E, H, F) / F ** 0.5, 128)
    logits = rand(T, E) + 0.5 * rand(E)
    logits[:, E // 2] = -math.inf
    logits[torch.rand(T, generator=g, device="cuda") < masked] = -math.inf
    routes = sd.route(logits, min(k, E - 1))
    r = rand(T, H).to(dt) if residual else None
    _say("experts", dtype, kind, T, H, F, E, k)
    got = sd.experts_forward(a, sa, routes, w1, s1, w2, s2, H, F, residual=r, dtype=dt).double()
    x, want = _values(torch, a, sa, 1, H), torch.zeros(T, H, dtype=torch.float64, device="cuda")
    if residual:
        want += r.double()
    assert int((routes.ids == E // 2).sum()) == 0
    for e in range(E):
        t, j = (routes.ids == e).nonzero(as_tuple=True)
        gate, more = (x[t] @ _values(torch, w1[e, i], s1[e, i], 128, H).t() for i in (0, 1))
        q = _rounded8(torch, gate * torch.sigmoid(gate) * more) if t.numel() else gate
        o = q @ _values(torch, w2[e], s2[e], 128, F).t()
        want.index_add_(0, t, o * routes.weight[t, j].double()[:, None])
    off, size = float((got - want).norm()), float(want.norm())
    if dtype == F32:
        assert off <= 1e-3 * size
    else:
        rounding = float((want.bfloat16().double() - want).norm())
        most = 1.03 if kind[0] == 64 else 1.45 if residual else 1.7
        assert off <= most * rounding, off / rounding
    dead = (routes.ids < 0).all(dim=1)
    assert torch.equal(got[dead], r.double()[dead] if residual else torch.zeros_like(got[dead]))
