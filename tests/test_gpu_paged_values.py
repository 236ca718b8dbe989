"""Values that are not finite under weights of any size: what a row sees makes its channel infinite or NaN, whatever rounding makes of the weight."""
import math

import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from test_gpu_paged import _attend, _compare, say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("depth", [0, 30, 60, 95])
@pytest.mark.parametrize("requests,hq,hkv,D", [([(700, 100, 0, 0)], 2, 1, 64),                    # tiles whose keys are cut
                                               ([(300, 130, 0, 0), (9, 1, 0, 0)], 3, 1, 128),     # tiles in one range, and a single row
                                               ([(0, 400, 0, 0)], 1, 1, 128),                     # a prompt
                                               ([(200, 40, 3, 20), (100, 30, 0, 0)], 2, 2, 64),   # branches in tiles, a team's rows beside them
                                               ([(150, 1, 3, 4)], 2, 1, 128)])                    # rows through the registers
def test_infinite_values_under_small_weights(requests, hq, hkv, D, depth, dtype):
    """Some slots' scores lie `depth` below the others (weights of e^-depth: zero in fp16 from 30 on, in bf16 at 95), and their values hold infinities
    and NaN in channels of their own: alone, of both signs, in blocks that all rows see and at the edge of what a row sees."""
    page, t = 32, U.TYPES[dtype]
    first = requests[0]
    total = first[0] + U.new_rows(first)
    # (slot, channel, value): no channel of them is touched by anything else
    odd = [(5, 3, math.inf), (40, 11, -math.inf), (40, 12, math.nan), (77, 20, math.inf), (101, 20, -math.inf), (total - 1, 30, math.inf), (total // 2, 31, -math.inf)]

    def poison(cache, lines, q):
        keys, values = cache.key_pages[-1].view(t), cache.value_pages[-1].view(t)
        ik, iv = U.offsets(D, page, "k").to(DEV), U.offsets(D, page, "v").to(DEV)
        for r, line in enumerate(lines):  # scores get scale * q0 * k0 = k0
            for s in range(len(line) * page):
                keys[line[s // page], :, ik[s % page][0]] = 0.0
        q.view(-1, q.shape[-1])[:, ::D] = math.sqrt(D) if D == 64 else 11.3125
        for s, d, value in odd:
            keys[lines[0][s // page], :, ik[s % page][0]] = -float(depth)
            values[lines[0][s // page], 0, iv[s % page][d]] = value

    say(requests, depth, dtype)
    cache, lines, q, out = _attend(requests, hq, hkv, D, dtype, page, poison=poison)
    rows = sum(map(U.new_rows, requests))
    see = U.visible(first).to(DEV)
    code = torch.zeros((rows, hq, D), device=DEV)
    for s, d, value in odd:
        seen = see[:, s]
        code[:U.new_rows(first), :hq // hkv, d] += torch.where(seen, value, 0.0)[:, None]
    clean = code == 0
    _compare(requests, cache, lines, q, out, hq, hkv, D, dtype, where=clean)
    got = out[:rows, :hq * D].reshape(rows, hq, D).float()
    assert torch.equal(torch.where(clean, 0.0, got).nan_to_num(7.0, 1.0, -1.0), code.nan_to_num(7.0, 1.0, -1.0))


@pytest.mark.parametrize("D", [64, 128])
def test_infinite_scores_stay_not_a_number(D):
    """An infinite query makes its row NaN, in channels with infinite values too, and leaves the rows beside it alone."""
    requests, t = [(300, 100, 0, 0)], torch.bfloat16

    def poison(cache, lines, q):
        q[7, :D] = math.inf
        cache.value_pages[0].view(t)[lines[0][0], 0, U.offsets(D, 32, "v")[5][9]] = math.inf

    cache, lines, q, out = _attend(requests, 2, 1, D, "bf16", 32, poison=poison)
    got = out[:100, :2 * D].reshape(100, 2, D)
    assert torch.isnan(got[7, 0]).all()
    rest = torch.ones((100, 2, D), dtype=torch.bool, device=DEV)
    rest[7, 0] = False
    assert torch.isposinf(got[:, :, 9][rest[:, :, 9]]).all()
    rest[:, :, 9] = False
    assert torch.isfinite(got[rest]).all()
