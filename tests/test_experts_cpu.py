"""Refusals of the operators of a layer of experts, and their sizes, without a GPU: no call here reaches a kernel."""

import ctypes
import math

import numpy as np
import pytest

from tests import blocks_ref as ref

FAKE = 1 << 20  # an aligned non-null address


@pytest.fixture(scope="module")
def sd():
    import paper_1708_02937_amd as sd

    return sd


def test_pitches(sd):
    for k, p, s in ((1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (513, 640, 8), (4096, 4096, 32)):
        assert sd.sdnn_blocks_pitch(k) == p and sd.sdnn_blocks_scale_pitch(k) == s
    for k in (0, -5, 1 << 31):
        assert sd.sdnn_blocks_pitch(k) == 0 and sd.sdnn_blocks_scale_pitch(k) == 0


def _status(sd, f, *args):
    try:
        f(*args)
        return 0
    except sd.SdnnError as e:
        return e.status


def _refusals(sd, f, good, changes):
    """f(**good) with each change alone is refused with that status, and nothing is launched."""
    for change, status in changes:
        args = dict(good)
        args.update(change)
        assert _status(sd, f, *args.values()) == status, (f.__name__, change)


def test_quantize_refusals(sd):
    good = dict(count=1, rows=2, k=3, block_rows=1, type=0, x=FAKE, ldx=3, codes=FAKE, scales=FAKE)
    _refusals(sd, sd.sdnn_quantize_blocks, good, [
        (dict(count=-1), 2), (dict(rows=-1), 2), (dict(k=0), 2), (dict(k=1 << 31), 2), (dict(block_rows=2), 2),
        (dict(type=2), 2), (dict(x=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(ldx=2), 2),
        (dict(x=FAKE + 2), 2), (dict(codes=FAKE + 8), 2), (dict(scales=FAKE + 1), 2)])
    assert _status(sd, sd.sdnn_quantize_blocks, 0, 2, 3, 1, 0, None, 3, None, None) == 0
    assert _status(sd, sd.sdnn_quantize_blocks, 1, 0, 3, 1, 0, None, 3, None, None) == 0


def test_norm_refusals(sd):
    good = dict(rows=2, k=8, type=1, x=FAKE, ldx=8, residual=FAKE, ldr=8, gamma=FAKE, eps=1e-6, sum=FAKE, lds=8,
                normed=FAKE, ldn=8, codes=FAKE, scales=FAKE)
    _refusals(sd, sd.sdnn_norm_quantize, good, [
        (dict(rows=-1), 2), (dict(k=0), 2), (dict(k=32769, ldx=40000, ldr=40000, lds=40000, ldn=40000), 9),
        (dict(type=-1), 2), (dict(eps=-1.0), 2), (dict(eps=math.nan), 2), (dict(eps=math.inf), 2),
        (dict(residual=None), 2), (dict(x=None), 1), (dict(gamma=None), 1), (dict(codes=None), 1),
        (dict(ldx=7), 2), (dict(ldr=7), 2), (dict(lds=7), 2), (dict(ldn=7), 2), (dict(gamma=FAKE + 2), 2),
        (dict(x=FAKE + 1), 2), (dict(codes=FAKE + 4), 2)])
    assert _status(sd, sd.sdnn_norm_quantize, 0, 8, 1, None, 8, None, 0, None, 1e-6, None, 0, None, 0, None, None) == 0


def test_product_refusals(sd):
    good = dict(m=2, n=3, k=4, a=FAKE, a_scale=FAKE, w=FAKE, w_scale=FAKE, bias=FAKE, activate=1, ymax=1.0, type=0,
                y=FAKE, ldy=3)
    _refusals(sd, sd.sdnn_product_blocks, good, [
        (dict(m=-1), 2), (dict(n=-1), 2), (dict(k=0), 2), (dict(a=None), 1), (dict(a_scale=None), 1),
        (dict(w=None), 1), (dict(w_scale=None), 1), (dict(y=None), 1), (dict(activate=2), 2), (dict(ymax=0.0), 2),
        (dict(ymax=math.nan), 2), (dict(type=7), 2), (dict(ldy=2), 2), (dict(a=FAKE + 8), 2),
        (dict(w_scale=FAKE + 2), 2), (dict(bias=FAKE + 2), 2), (dict(y=FAKE + 2), 2)])
    assert _status(sd, sd.sdnn_product_blocks, 0, 3, 4, None, None, None, None, None, 0, 0.0, 0, None, 3) == 0


def test_route_refusals(sd):
    good = dict(tokens=5, experts=12, chosen=3, score=0, type=0, logits=FAKE, ldl=12, bias=FAKE, groups=4,
                groups_kept=2, group_best=2, normalize=1, factor=1.0, ids=FAKE, weight=FAKE, offsets=FAKE, order=FAKE,
                ws=FAKE, ws_bytes=1 << 30)
    _refusals(sd, sd.sdnn_route, good, [
        (dict(tokens=-1), 2), (dict(experts=0), 2), (dict(chosen=0), 2), (dict(chosen=13), 2),
        (dict(experts=1025, ldl=1025, groups=1, groups_kept=1), 9), (dict(experts=1000, chosen=65, ldl=1000), 9),
        (dict(tokens=1 << 30), 9), (dict(score=2), 2), (dict(type=3), 2), (dict(groups=5), 2), (dict(groups=0), 2),
        (dict(groups_kept=5), 2), (dict(groups_kept=0), 2), (dict(group_best=3), 2), (dict(normalize=2), 2),
        (dict(factor=math.inf), 2), (dict(logits=None), 1), (dict(ids=None), 1), (dict(weight=None), 1),
        (dict(offsets=None), 1), (dict(order=None), 1), (dict(ldl=11), 2), (dict(bias=FAKE + 1), 2),
        (dict(ids=FAKE + 2), 2), (dict(ws_bytes=-1), 6), (dict(ws=FAKE + 4), 2)])


def test_experts_refusals(sd):
    good = dict(tokens=3, width=10, inner=20, experts=4, chosen=2, a=FAKE, a_scale=FAKE, ids=FAKE, weight=FAKE,
                offsets=FAKE, order=FAKE, w_in=FAKE, w_in_scale=FAKE, w_out=FAKE, w_out_scale=FAKE, type=1,
                residual=FAKE, ldr=10, out=FAKE, ldo=10, ws=FAKE, ws_bytes=1 << 30)
    changes = [(dict(tokens=-1), 2), (dict(width=0), 2), (dict(inner=0), 2), (dict(chosen=5), 2), (dict(type=9), 2),
               (dict(ldr=9), 2), (dict(ldo=9), 2), (dict(ws=None), 1), (dict(ws_bytes=100), 6),
               (dict(ws=FAKE + 8), 2), (dict(order=FAKE + 1), 2)]
    changes += [({x: None}, 1) for x in ("a", "a_scale", "ids", "weight", "offsets", "order", "w_in", "w_in_scale",
                                         "w_out", "w_out_scale", "out")]
    changes += [({x: FAKE + 8}, 2) for x in ("a", "w_in", "w_out")]
    _refusals(sd, sd.sdnn_experts_forward, good, changes)
    assert "ws" in (_status(sd, sd.sdnn_experts_forward, *{**good, "ws": None}.values()) and sd.sdnn_last_error())


def test_workspace_sizes(sd):
    out = ctypes.c_int64()
    assert sd.lib.sdnn_route_workspace_size(5, 4, 2, None) == 1
    assert sd.lib.sdnn_experts_workspace_size(5, 8, 8, 4, 2, 0, None) == 1
    assert sd.lib.sdnn_experts_workspace_size(5, 8, 8, 4, 9, 0, ctypes.byref(out)) == 2
    small = sd.sdnn_experts_workspace_size(1, 256, 128, 8, 2, 1)
    large = sd.sdnn_experts_workspace_size(64, 256, 128, 8, 2, 1)
    # at least the slots' inner rows (8 bits) and output rows (bfloat16)
    assert small >= 2 * 128 and large >= 64 * 2 * 128 and large > small


def test_tensors_on_the_host_are_refused(sd):
    import torch

    x = torch.zeros(2, 8)
    for call in (lambda: sd.norm_quantize(x, x[0]), lambda: sd.route(x, 1), lambda: sd.quantize_blocks(x)):
        with pytest.raises(ValueError):
            call()


def test_reference_codes():
    """The reference's table and rounding: known values of the 8-bit type, every code its own, ties to even."""
    assert ref.TABLE[0x7E] == 448 and ref.TABLE[0x01] == 2.0 ** -9 and ref.TABLE[0x38] == 1.0
    assert np.isnan(ref.TABLE[[0x7F, 0xFF]]).all() and ref.TABLE[0xB8] == -1.0
    finite = np.array([c for c in range(256) if c & 127 != 127])
    assert np.array_equal(ref.encode(ref.TABLE[finite]), finite)
    assert list(ref.encode(np.array([1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]))) == [0x38, 0x3A, 0x00, 0x02]
    q, s = ref.quantize(np.array([[448.0, 1.0], [448.5, 1.0]]))
    assert list(s[:, 0]) == [127, 128] and list(q[:, 1]) == [0x38, 0x30]
