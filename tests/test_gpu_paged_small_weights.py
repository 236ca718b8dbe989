"""One key in front of a long flat tail: the weights of the tail are small each, and what they add up to is in the output."""
import math

import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from test_gpu_paged import _attend, say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("gap", [9.0, 17.625, 20.0])
@pytest.mark.parametrize("request_,hq,hkv,page", [((9000, 1, 0, 0), 2, 2, 64), ((9000, 20, 0, 0), 2, 1, 64), ((700, 40, 0, 0), 1, 1, 32),  # rows through registers, teams
                                                  ((9000, 80, 0, 0), 2, 1, 64), ((7000, 2048, 0, 0), 16, 16, 256)])  # tiles: keys cut, and in one range
def test_a_tail_below_one_key(request_, hq, hkv, page, gap, dtype):
    """Key 0 scores `gap`, all others 0: weights of e^-gap, 2^-13 to 2^-29, of the largest."""
    D, t = 64, U.TYPES[dtype]
    gap = float(torch.tensor(gap, dtype=t))  # the score as the type holds it: 8 * gap / sqrt(64)

    def poison(cache, lines, q):
        keys, values = cache.key_pages[0].view(t), cache.value_pages[0].view(t)
        keys.zero_()
        keys[lines[0][0], :, U.offsets(D, page, "k")[0][0]] = gap
        values.copy_(torch.rand(values.shape, generator=torch.Generator().manual_seed(1)) * 0.5 + 0.5)
        values[lines[0][0], :, U.offsets(D, page, "v")[0].to(DEV)] = 0.0
        q.zero_()
        q[:, ::D] = 8.0

    cache, lines, q, out = _attend([request_], hq, hkv, D, dtype, page, poison=poison)
    rows, keys = U.new_rows(request_), request_[0] + U.new_rows(request_)
    V = U.rows_of(cache.value_pages[0].view(t), lines[0], D, "v")[:, :keys].double()
    sums = V.cumsum(1)[:, request_[0]:].transpose(0, 1)  # [rows][kv heads][D]: key 0's values are zero
    count = torch.arange(request_[0], keys, device=DEV, dtype=torch.float64)[:, None, None]  # keys behind the first that a row sees
    want = (sums * math.exp(-gap) / (1.0 + count * math.exp(-gap))).repeat_interleave(hq // hkv, 1)
    got = out[:rows, :hq * D].reshape(rows, hq, D).double()
    # With u half a step of the type: the output is rounded once; a weight once (u) or as a pair (u^2), and in fp16, where the smallest weights lie
    # on a grid of 2^-24 after they were raised by 2^7, off by up to 2^-32 of the largest weight each; exponents are fp32 (2^-23 of up to 2 * 20 + 16),
    # sums over the keys too.  A relative error of the weights moves numerator and sum.
    u = torch.finfo(t).eps / 2
    pairs = rows * (hq // hkv) <= 64
    e = (u * u if pairs else u) + 2.0 ** -23 * 56 + keys * 2.0 ** -23
    bound = u * want * (1 + u) + (1 + u) * (2 * e * want + (keys * 2.0 ** -32 if dtype == "fp16" else 0.0))
    err = (got - want).abs()
    say(request_, gap, dtype, "largest error over bound", float((err / bound).max()), "largest output", float(want.max()))
    assert (err <= bound).all()
