"""A request whose cached tokens hold no pages yet: the plan gives it pages for them, and the caller writes what they hold."""
import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from paper_2503_00784_amd import binding as B
from test_gpu_paged import _compare

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("held", [0, 1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_prefix_that_is_brought_back(dtype, held):
    requests, hq, hkv, D, page, t = [(40, 1, 0, 0), (90, 1, 1, 3), (0, 70, 0, 0)], 4, 2, 64, 32, U.TYPES[dtype]
    cache, lines = U.make(requests, hq, hkv, D, dtype, page, seed=held)
    free = [p for p in range(cache.n_pages) if p not in lines[0] and p not in lines[1][:held] and p not in lines[2]]
    U.set_tables(cache, [lines[0], lines[1][:held], lines[2]], free)
    cache.plan()
    assert cache.status.item() == 0 and cache.tables.held.tolist() == [2, 3, 3]
    got = [line[:n] for line, n in zip(cache.tables.block_table.tolist(), (2, 3, 3))]
    assert got[0] == lines[0] and got[2] == lines[2] and got[1] == lines[1][:held] + free[::-1][:3 - held]
    assert len({p for line in got for p in line}) == 8
    g = torch.Generator(device=DEV).manual_seed(held)
    for kind, pool in (("k", cache.key_pages), ("v", cache.value_pages)):  # the prefix from outside, by the map of the cache's tiles
        idx = U.offsets(D, page, kind).to(DEV)
        s = torch.arange(90, device=DEV)
        pid = torch.tensor(got[1], device=DEV)[s // page]
        for h in range(hkv):
            pool[0].view(t)[pid[:, None], h, idx[s % page]] = torch.randn((90, D), generator=g, device=DEV).to(t)
    q, k, v = ((torch.randn((cache.max_rows, h, D), generator=g, device=DEV) * 1.28).to(t) for h in (hq, hkv, hkv))
    cache.append(0, q, k, v)
    out = torch.full((cache.max_rows, hq * D), 9.0, dtype=t, device=DEV)
    cache.attention(0, q, out)
    _compare(requests, cache, got, q, out, hq, hkv, D, dtype)
    cache.commit(torch.tensor([[-1, 0, 1, 0], [0, 2, 1, 0], [-1, 0, 1, 0]], dtype=torch.int32, device=DEV))
    assert cache.cached.tolist() == [41, 93, 70] and cache.status.item() == 0
