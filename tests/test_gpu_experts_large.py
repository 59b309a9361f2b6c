"""The layer of experts where offsets pass 32 bits: rows on both sides of the places where an offset in elements or bytes
passes 2^31 and 2^32, and the last ones, are those of a call on these rows alone, bit for bit."""

import pytest

pytestmark = pytest.mark.gpu

ROWS, K = (1 << 20) + 300, 4096  # 4.3e9 codes


@pytest.fixture(scope="module")
def torch():
    import torch

    yield torch
    torch.cuda.empty_cache()


@pytest.fixture(scope="module")
def sd():
    import paper_1708_02937_amd as sd

    return sd


def _say(*a):
    print("[case]", *a, flush=True)


def _places(rows, *row_bytes):
    """Starts of runs of 256 rows (multiples of 128), around offsets of 2^31 and 2^32 and at the end."""
    at = {rows - 256 - rows % 128, 0}
    for size in row_bytes:
        for limit in (1 << 31, 1 << 32):
            if limit // size < rows:
                at.add(max(0, limit // size // 128 * 128 - 128))
    return sorted(at)


def _same(torch, a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_norm_and_rounding(torch, sd):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(ROWS, K, generator=g, device="cuda", dtype=torch.bfloat16)
    gamma = 1 + 0.1 * torch.randn(K, generator=g, device="cuda")
    _say("norm", ROWS, K)
    full = sd.norm_quantize(x, gamma, residual=x, normed=True)
    for p in _places(ROWS, K, 2 * K):
        part = sd.norm_quantize(x[p:p + 256], gamma, residual=x[p:p + 256], normed=True)
        for u, v in zip(full, part):
            assert _same(torch, u[p:p + 256], v), p
    del full
    for block_rows in (1, 128):
        _say("quantize", ROWS, K, block_rows)
        codes, scales = sd.quantize_blocks(x, block_rows)
        for p in _places(ROWS, K, 2 * K):
            c, s = sd.quantize_blocks(x[p:p + 256].clone(), block_rows)
            assert _same(torch, codes[p:p + 256], c), p
            assert _same(torch, scales[p // block_rows:(p + 256) // block_rows], s), p


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_product(torch, sd, dtype):
    """Many rows, and many outputs of few rows (small integers: exact)."""
    g = torch.Generator(device="cuda").manual_seed(2)
    dt = getattr(torch, dtype)
    big, sb = sd.quantize_blocks(torch.randint(-2, 3, (ROWS, K), generator=g, device="cuda", dtype=torch.int8).bfloat16())
    few = torch.randint(-2, 3, (33, K), generator=g, device="cuda").float()
    w, sw = sd.quantize_blocks(few, 128)
    _say("product", ROWS, K, dtype)
    y = sd.product_blocks(big, sb, w, sw, K, dtype=dt)
    for p in _places(ROWS, K):
        assert torch.equal(y[p:p + 256], (big[p:p + 256].float() * _scale(torch, sb[p:p + 256]) @ few.t()).to(dt)), p
    # the same matrix as weights: every block's largest value is 2, so its rows share a scale
    a, sa = sd.quantize_blocks(few)
    same = sb.view(torch.uint8).unflatten(1, (-1, 4)).amax()
    assert bool((sb.view(torch.uint8)[:, :K // 128] == same).all())
    rows = ROWS // 128 * 128
    _say("product of many outputs", rows, K, dtype)
    y = sd.product_blocks(a, sa, big[:rows], sb[:rows:128].contiguous(), K, dtype=dt)
    for p in _places(rows, K):
        want = few @ (big[p:p + 256].float() * _scale(torch, sb[p:p + 256])).t()
        assert torch.equal(y[:, p:p + 256], want.to(dt)), p


def _scale(torch, s):
    """The powers of two of a whole matrix whose blocks have one scale."""
    return float(torch.exp2(s.view(torch.uint8)[0, 0].double() - 127))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,H,F", [(300_000, 128, 4096), (300_000, 2048, 128)])
def test_experts(torch, sd, T, H, F, dtype):
    """The slots' inner rows (4.9e9 codes), and their outputs (2.5e9 values), past 32 bits; a part of the tokens is enough
    for the same kernels."""
    E, k, part = 6, 4, 40_000
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = getattr(torch, dtype)
    a, sa = sd.quantize_blocks(rand(T, H))
    weights = (*sd.quantize_blocks(rand(E, 2, F, H) / H ** 0.5, 128), *sd.quantize_blocks(rand(E, H, F) / F ** 0.5, 128))
    logits = rand(T, E)
    _say("experts", T, H, F, dtype)
    out = sd.experts_forward(a, sa, sd.route(logits, k), *weights, H, F, dtype=dt)
    for p in (0, T // 2, T - part):
        at = slice(p, p + part)
        want = sd.experts_forward(a[at], sa[at], sd.route(logits[at], k), *weights, H, F, dtype=dt)
        assert torch.equal(out[at], want), p
