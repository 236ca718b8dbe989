"""The rows that append and attention may share: fused projections with the rotated queries in place or beside them."""
import pytest

torch = pytest.importorskip("torch")

import paged_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("requests", [[(5, 1, 0, 0)], [(40, 1, 2, 3), (0, 37, 0, 0)]])
def test_outputs_in_the_matrix_of_the_inputs(requests, pad):
    """q | k | v | output: every place of the output gives what matrices of their own give."""
    hq, hkv, D = 4, 2, 64
    cache, _ = U.make(requests, hq, hkv, D, "bf16", 32, pad=pad)
    cache.plan()
    g = torch.Generator(device=DEV).manual_seed(3)
    fused = torch.randn((cache.max_rows, (2 * hq + 2 * hkv) * D), generator=g, device=DEV).bfloat16()
    cuts = (hq * D, hkv * D, hkv * D, hq * D)
    q, k, v, _ = (x.contiguous() for x in fused.split(cuts, 1))
    pools = [cache.key_pages.clone(), cache.value_pages.clone()]
    want_q = cache.append(0, q, k, v, torch.zeros_like(q))
    want_out = cache.attention(0, want_q, torch.zeros_like(q))
    want_pools = [cache.key_pages.clone(), cache.value_pages.clone()]
    rows = cache.row_start[-1].item()
    for place in (0, 3):
        for pool, was in zip((cache.key_pages, cache.value_pages), pools):
            pool.copy_(was)
        x = fused.clone()
        parts = x.split(cuts, 1)
        turned = cache.append(0, *parts[:3], parts[place])
        assert torch.equal(turned[:rows], want_q[:rows]) and torch.equal(turned[rows:], fused.split(cuts, 1)[place][rows:])
        assert torch.equal(cache.key_pages, want_pools[0]) and torch.equal(cache.value_pages, want_pools[1])
        out = parts[3 - place]
        cache.attention(0, turned, out)
        assert torch.equal(out[:rows], want_out[:rows]) and cache.status.item() == 0
