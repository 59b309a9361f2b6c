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
