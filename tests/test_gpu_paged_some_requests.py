"""Whole steps of the first requests of a cache, and matrices given as bit patterns."""
import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from test_gpu_paged import _compare

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
REQUESTS = [(40, 1, 2, 3), (0, 50, 0, 0), (70, 1, 0, 0), (300, 1, 1, 9), (33, 40, 2, 20), (10, 1, 1, 2), (64, 1, 0, 0), (0, 9, 0, 0), (5, 0, 2, 2), (90, 1, 3, 3)]


@pytest.mark.parametrize("count", [1, 2, 5, 8, 9])
def test_a_step_of_some_requests(count):
    """Requests behind the planned ones keep their pages, their keys and values and their lengths."""
    hq, hkv, D, dtype, page, t = 4, 2, 64, "bf16", 32, torch.bfloat16
    cache, lines = U.make(REQUESTS, hq, hkv, D, dtype, page, layers=2)
    mine = REQUESTS[:count]
    rows = sum(map(U.new_rows, mine))
    cache.plan(count)
    assert cache.status.item() == 0 and cache.row_start[count].item() == rows and (cache.slot[rows:] == -1).all()
    others = torch.tensor([p for line in lines[count:] for p in line], device=DEV)
    before = [pool[:, others].clone() for pool in (cache.key_pages, cache.value_pages)]
    g = torch.Generator(device=DEV).manual_seed(count)
    q, k, v = ((torch.randn((cache.max_rows, h, D), generator=g, device=DEV) * 1.28).to(t) for h in (hq, hkv, hkv))
    cache.append(1, q, k, v)
    out = torch.full((cache.max_rows, hq * D), 9.0, dtype=t, device=DEV)
    cache.attention(1, q, out)
    _compare(mine, cache, lines, q, out, hq, hkv, D, dtype)
    records = [[n - 1, k, 3, 0] if n * k else [-1, 0, 3, 0] for _, _, n, k in mine]
    cache.commit(torch.tensor(records, dtype=torch.int32, device=DEV))
    assert cache.status.item() == 0
    assert cache.cached.tolist() == [c + trunk + (k if n * k else 0) for c, trunk, n, k in mine] + [r[0] for r in REQUESTS[count:]]
    for pool, was in zip((cache.key_pages, cache.value_pages), before):
        assert torch.equal(pool[:, others], was)
    assert cache.tables.held.tolist() == [len(line) for line in lines]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_bit_patterns(dtype):
    """int16 matrices, alone or beside typed ones, give the bits of typed ones."""
    hq, hkv, D, t = 4, 2, 128, U.TYPES[dtype]
    cache, _ = U.make(REQUESTS, hq, hkv, D, dtype, 32)
    cache.plan()
    q, k, v = ((torch.randn((cache.max_rows, h, D), device=DEV) * 1.28).to(t) for h in (hq, hkv, hkv))
    typed = cache.append(0, q, k, v, torch.zeros_like(q))
    pools = [cache.key_pages.clone(), cache.value_pages.clone()]
    want = cache.attention(0, typed)
    bits = cache.append(0, q.view(torch.int16), k.view(torch.int16), v, torch.zeros_like(q).view(torch.int16))
    assert torch.equal(bits, typed.view(torch.int16)) and torch.equal(pools[0], cache.key_pages) and torch.equal(pools[1], cache.value_pages)
    got = cache.attention(0, bits)
    assert got.dtype == torch.int16 and torch.equal(got, want.view(torch.int16))
    assert torch.equal(cache.attention(0, bits, torch.zeros_like(want)), want)
