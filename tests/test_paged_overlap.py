"""Outputs of the paged-cache calls that share elements with what other workgroups still read are refused, column ranges of one matrix
are not.  No GPU: nothing is enqueued."""
import ctypes as C
import itertools

import pytest

from paper_2503_00784_amd import binding as B
from paper_2503_00784_amd import inputs

HQ, HKV, D = 4, 2, 64
QD, KD = HQ * D, HKV * D
BASE = 0x100000
ROWS = 6


def _args(max_rows=ROWS):
    cfg = B.make_config(inputs.ModelShape(1, 64 * HQ, HQ, HKV, D, 64, 1000), 32)
    return cfg, B.PageCacheC(0x1000, 0x1000, 10, 64, 4), B.PageBatchC(*[0x1000] * 8, 3, max_rows, max_rows)


def _attention(q, out, rows=ROWS):
    """The call's code with a workspace that is too small, so that nothing is enqueued: -8 refused for its rows, -5 for the workspace."""
    cfg, cache, batch = _args(rows)
    return B.load().duo_page_attention(C.byref(cfg), C.byref(cache), 0x1000, C.byref(batch), 0, *q, *out, 0.0, 0x1000, 0, None)


def _append(q, k, v, q_out, rows=ROWS):
    cfg, cache, batch = _args(rows)
    return B.load().duo_page_append(C.byref(cfg), C.byref(cache), C.byref(batch), 0, *q, *k, *v, *q_out, None)


def at(elements, stride):
    return BASE + 2 * elements, stride


def _elements(start, stride, width, rows):
    return {start + i * stride + j for i in range(rows) for j in range(0, width, 8)}  # everything is a multiple of 8 elements


@pytest.mark.parametrize("rows", [1, 2, ROWS])
def test_attention_tells_column_ranges_apart(rows):
    """Every offset of the output from the queries, in steps of eight elements, against the sets of their elements."""
    stride = QD + 40
    far = _elements(0, stride, QD, rows)
    for offset in range(-(rows + 1) * stride, (rows + 1) * stride + 8, 8):
        q = BASE // 2 + (rows + 2) * stride
        q -= q % 8
        got = _attention((2 * q, stride), (2 * (q + offset), stride), rows)
        meets = bool(far & _elements(offset, stride, QD, rows))
        assert got == (-8 if meets else -5), (offset, got)


def test_attention_of_other_distances_goes_by_address():
    q, wide = at(0, QD), 2 * QD
    end = (ROWS - 1) * QD + QD
    for offset, code in ((end, -5), (end - 8, -8), (0, -8), (-(ROWS - 1) * wide - QD, -5), (-(ROWS - 1) * wide - QD + 8, -8)):
        assert _attention(q, at(offset, wide)) == code, offset


def test_append_refuses_outputs_over_its_inputs():
    """Fused rows q | k | v | rest: the rotated queries may go in place or to the rest, nowhere else."""
    stride = 2 * QD + 2 * KD
    q, k, v = at(0, stride), at(QD, stride), at(QD + KD, stride)
    for offset in (8, 64, QD - 8, QD, QD + KD - 8, QD + KD, QD + 2 * KD - 8, -8, stride, stride - 8, (ROWS - 1) * stride + 8, -(ROWS - 1) * stride):
        assert _append(q, k, v, at(offset, stride)) == -8, offset
    for offset in (QD, 0):  # over k and over q, by rows of another distance
        assert _append(q, k, v, at(offset, QD)) == -8, offset
    apart = at(100 * stride, KD)
    for one, other in itertools.permutations((k, v), 2):  # one of them alone meets the output
        assert _append(at(200 * stride, QD), one, apart, one[:1] + (stride,)) == -8
        assert _append(at(200 * stride, QD), apart, one, one[:1] + (stride,)) == -8
