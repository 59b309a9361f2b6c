"""Refusals of the operators that generate tokens, and their sizes, without a GPU: no call here reaches a kernel."""

import math

import numpy as np
import pytest

from tests import generate_ref as gen
from tests.test_experts_cpu import FAKE, _refusals, _status, sd  # noqa: F401  (the last is a fixture)


def test_pitches(sd):  # noqa: F811
    for k, p, s in ((1, 64, 4), (128, 64, 4), (129, 128, 8), (4096, 2048, 128)):
        assert sd.sdnn_groups_pitch(k) == p and sd.sdnn_groups_scale_pitch(k) == s
    for k in (0, -5, 1 << 31):
        assert sd.sdnn_groups_pitch(k) == 0 and sd.sdnn_groups_scale_pitch(k) == 0


def test_quantize_and_widen_refusals(sd):  # noqa: F811
    good = dict(rows=2, k=3, type=0, x=FAKE, ldx=3, codes=FAKE, scales=FAKE)
    _refusals(sd, sd.sdnn_quantize_groups, good, [
        (dict(rows=-1), 2), (dict(rows=1 << 31), 2), (dict(k=0), 2), (dict(k=1 << 31), 2), (dict(type=2), 2),
        (dict(x=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(ldx=2), 2), (dict(x=FAKE + 2), 2),
        (dict(codes=FAKE + 8), 2), (dict(scales=FAKE + 2), 2)])
    assert _status(sd, sd.sdnn_quantize_groups, 0, 3, 0, None, 3, None, None) == 0
    good = dict(rows=2, k=3, codes=FAKE, scales=FAKE, type=1, y=FAKE, ldy=3)
    _refusals(sd, sd.sdnn_widen_groups, good, [
        (dict(rows=-1), 2), (dict(k=0), 2), (dict(type=-1), 2), (dict(y=None), 1), (dict(codes=None), 1),
        (dict(scales=None), 1), (dict(ldy=2), 2), (dict(y=FAKE + 1), 2), (dict(codes=FAKE + 4), 2)])
    assert _status(sd, sd.sdnn_widen_groups, 0, 3, None, None, 1, None, 3) == 0


def test_product_refusals(sd):  # noqa: F811
    good = dict(m=2, n=3, k=4, x_type=0, x=FAKE, ldx=4, w=FAKE, w_scale=FAKE, bias=FAKE, activate=1, ymax=1.0, y_type=1,
                y=FAKE, ldy=3)
    _refusals(sd, sd.sdnn_product_groups, good, [
        (dict(m=-1), 2), (dict(n=-1), 2), (dict(k=0), 2), (dict(x_type=2), 2), (dict(y_type=2), 2), (dict(x=None), 1),
        (dict(w=None), 1), (dict(w_scale=None), 1), (dict(y=None), 1), (dict(activate=2), 2), (dict(ymax=0.0), 2),
        (dict(ymax=math.nan), 2), (dict(ldx=3), 2), (dict(ldy=2), 2), (dict(x=FAKE + 2), 2), (dict(w=FAKE + 8), 2),
        (dict(w_scale=FAKE + 2), 2), (dict(bias=FAKE + 2), 2), (dict(y=FAKE + 1), 2)])
    assert _status(sd, sd.sdnn_product_groups, 0, 3, 4, 0, None, 4, None, None, None, 0, 0.0, 0, None, 3) == 0
    assert _status(sd, sd.sdnn_product_groups, 2, 0, 4, 0, None, 4, None, None, None, 0, 0.0, 0, None, 3) == 0


def test_tensors_on_the_host_are_refused(sd):  # noqa: F811
    import torch

    x = torch.zeros(2, 8)
    w, s = torch.zeros(3, 64, dtype=torch.float4_e2m1fn_x2), torch.ones(3, 4).to(torch.float8_e8m0fnu)
    for call in (lambda: sd.quantize_groups(x), lambda: sd.widen_groups(w, s, 8), lambda: sd.product_groups(x, w, s)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_reference_codes():
    """The reference's rounding: known values, every code its own, ties to the even code."""
    assert np.array_equal(gen.encode4(gen.TABLE), np.arange(16))
    assert list(gen.encode4(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, 5.1]))) == [0, 2, 2, 4, 4, 6, 6, 1, 7]
    codes, scales = gen.quantize4(np.array([[6.0, 3.0, 6.1], [-6.0, 0.0, 0.0]]))
    assert scales[0, 0] == 128 and scales[1, 0] == 127 and codes[0, 0] == 5 | 3 << 4 and codes[1, 0] == 15
    assert np.array_equal(gen.values4(codes, scales, 3), [[6.0, 3.0, 6.0], [-6.0, 0.0, 0.0]])


def test_layer_refusals(sd):  # noqa: F811
    good = dict(tokens=3, width=10, inner=20, experts=4, chosen=2, type=1, x=FAKE, ldx=10, residual=FAKE, ldr=10,
                gamma=FAKE, eps=1e-6, live=FAKE + 1, router_type=0, router=FAKE, ldw=10, score=1, bias=FAKE, groups=2,
                groups_kept=1, group_best=2, normalize=1, factor=1.0, w_in=FAKE, w_in_scale=FAKE, w_out=FAKE,
                w_out_scale=FAKE, out=FAKE, ldo=10, ids=FAKE, weight=FAKE, ws=FAKE, ws_bytes=1 << 30)
    changes = [(dict(tokens=-1), 2), (dict(tokens=17), 9), (dict(width=0), 2), (dict(inner=0), 2), (dict(experts=0), 2),
               (dict(width=1 << 27, ldx=1 << 28, ldr=1 << 28, ldw=1 << 28, ldo=1 << 28), 9), (dict(chosen=5), 2),
               (dict(chosen=0), 2), (dict(experts=1025, groups=1), 9), (dict(type=9), 2), (dict(router_type=2), 2),
               (dict(eps=-1.0), 2), (dict(eps=math.nan), 2), (dict(score=2), 2), (dict(groups=3), 2),
               (dict(groups_kept=3), 2), (dict(group_best=0), 2), (dict(normalize=2), 2), (dict(factor=math.inf), 2),
               (dict(ldx=9), 2), (dict(ldr=9), 2), (dict(ldw=9), 2), (dict(ldo=9), 2), (dict(x=FAKE + 1), 2),
               (dict(router=FAKE + 2), 2), (dict(gamma=FAKE + 2), 2), (dict(bias=FAKE + 1), 2), (dict(ids=FAKE + 2), 2),
               (dict(weight=FAKE + 2), 2), (dict(ws=None), 1), (dict(ws_bytes=100), 6), (dict(ws_bytes=-1), 6),
               (dict(ws=FAKE + 8), 2)]
    changes += [({x: None}, 1) for x in ("x", "gamma", "router", "w_in", "w_in_scale", "w_out", "w_out_scale", "out",
                                         "ids", "weight")]
    changes += [({x: FAKE + 8}, 2) for x in ("w_in", "w_out")]
    _refusals(sd, sd.sdnn_experts_layer, good, changes)
    none = {k: (None if v in (FAKE, FAKE + 1) else v) for k, v in good.items()}
    assert _status(sd, sd.sdnn_experts_layer, *{**none, "tokens": 0}.values()) == 0


def test_layer_workspace_sizes(sd):  # noqa: F811
    """One of the size for the most tokens serves every smaller call."""
    for width, inner, experts, chosen in ((1, 1, 1, 1), (300, 70, 8, 3), (4096, 1024, 64, 8), (100, 33, 1024, 64)):
        sizes = [sd.sdnn_experts_layer_workspace_size(t, width, inner, experts, chosen) for t in range(17)]
        assert sizes == sorted(sizes) and sizes[1] >= chosen * inner * 4 + width
    assert _status(sd, sd.sdnn_experts_layer_workspace_size, 17, 8, 8, 4, 2) == 9
    assert _status(sd, sd.sdnn_experts_layer_workspace_size, 1, 8, 8, 4, 5) == 2
    assert sd.lib.sdnn_experts_layer_workspace_size(1, 8, 8, 4, 2, None) == 1


def test_the_widest_layer(sd):  # noqa: F811
    """A launch holds fewer than 2^32 threads: 512 for each 16 columns are one too many from 2^27 - 15 columns on."""
    wide = (1 << 27) - 16
    assert wide // 16 * 512 < 1 << 32 <= (wide + 1 + 15) // 16 * 512
    assert sd.sdnn_experts_layer_workspace_size(1, wide, 8, 4, 2) > 0
    for width in (wide + 1, wide + 15, wide + 16):
        assert _status(sd, sd.sdnn_experts_layer_workspace_size, 1, width, 8, 4, 2) == 9


def test_sample_refusals(sd):  # noqa: F811
    good = dict(rows=3, vocab=40000, type=1, logits=FAKE, ldl=40000, uniform=FAKE, temperature=FAKE, top_k=FAKE,
                top_p=FAKE, min_p=FAKE, ids=FAKE, prob=FAKE, kept=FAKE, ws=FAKE, ws_bytes=1 << 30)
    changes = [(dict(rows=-1), 2), (dict(vocab=0), 2), (dict(vocab=1 << 31, ldl=1 << 31), 2), (dict(type=2), 2),
               (dict(ldl=39999), 2), (dict(logits=FAKE + 1), 2), (dict(uniform=FAKE + 4), 2), (dict(ws=None), 1),
               (dict(ws_bytes=100), 6), (dict(ws_bytes=-1), 6), (dict(ws=FAKE + 8), 2)]
    changes += [({x: None}, 1) for x in ("logits", "uniform", "ids", "prob", "kept")]
    changes += [({x: FAKE + 2}, 2) for x in ("temperature", "top_k", "top_p", "min_p", "ids", "prob", "kept")]
    _refusals(sd, sd.sdnn_sample, good, changes)
    assert _status(sd, sd.sdnn_sample, 0, 5, 0, None, 5, None, None, None, None, None, None, None, None, None, 0) == 0


def test_sample_workspace_sizes(sd):  # noqa: F811
    """One of the size for the most rows serves every smaller call."""
    for vocab in (1, 100, 16384, 16385, 32768, 32769, 50021, 131072, 10**6, 5 * 10**6, 2**31 - 1):
        sizes = [sd.sdnn_sample_workspace_size(r, vocab) for r in list(range(1100)) + [5000, 100000]]
        assert sizes == sorted(sizes) and (sizes[1] == 0) == (vocab <= 16384)
    assert _status(sd, sd.sdnn_sample_workspace_size, -1, 8) == 2
    assert _status(sd, sd.sdnn_sample_workspace_size, 1, 0) == 2
    assert sd.lib.sdnn_sample_workspace_size(1, 8, None) == 1


def test_reference_sample():
    """The reference by hand: four tokens of masses 8, 4, 2, 1 (in any order of the row)."""
    l = np.log(np.array([2.0, 8.0, 1.0, 4.0]))
    assert gen.sample(l, 0.0, 1.0, 0, 1.0, 0.0)[:3] == (0, pytest.approx(2 / 15), 4)
    assert gen.sample(l, 0.5, 1.0, 0, 1.0, 0.0)[0] == 1 and gen.sample(l, 0.99, 1.0, 0, 1.0, 0.0)[0] == 3
    assert gen.sample(l, 0.9, 1.0, 2, 1.0, 0.0)[:3] == (3, pytest.approx(4 / 12), 2)
    assert gen.sample(l, 0.9, 1.0, 0, 0.75, 0.0)[2] == 2 and gen.sample(l, 0.9, 1.0, 0, 0.85, 0.0)[2] == 3
    assert gen.sample(l, 0.9, 1.0, 0, 1.0, 0.2)[2] == 3 and gen.sample(l, 0.9, 0.0, 0, 1.0, 0.0)[:3] == (1, 1.0, 1)
    assert gen.sample(np.full(3, -np.inf), 0.9, 1.0, 0, 1.0, 0.0)[:3] == (-1, 0.0, 0)
