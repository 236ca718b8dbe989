"""The per-kernel timer sees the kernels of the paged-cache calls, each once and under its class."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# requests, launches of (plan, append, attention, joining of ranges, commit): short requests alone are not cut, more than eight requests are planned
# in two launches
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("requests,launches", [([(20, 1, 1, 3), (40, 1, 0, 0)], (1, 1, 1, 0, 1)), ([(2000, 1, 1, 3), (0, 100, 0, 0)], (1, 1, 1, 1, 1)),
                                               ([(r, 1, 1, 2) for r in range(9)], (2, 1, 1, 0, 1))])
def test_timer_counts_the_launches_of_a_paged_step(requests, launches, dtype):
    cache, _ = U.make(requests, 4, 2, 64, dtype, 32)
    q = torch.randn((cache.max_rows, 4, 64), device=DEV).to(U.TYPES[dtype])
    kv = q[:, :2].contiguous()
    records = torch.tensor([[-1, 0, 1, 0]] * len(requests), dtype=torch.int32, device=DEV)

    def step():
        cache.plan()
        cache.append(0, q, kv, kv)
        cache.attention(0, q, torch.empty_like(q))
        cache.commit(records, torch.zeros_like(cache.cached))

    step()
    torch.cuda.synchronize()
    B.profile_enable(True, dtype)
    try:
        step()
        assert B.profile_dropped(dtype) == 0
        prof = B.profile_read(dtype)
    finally:
        B.profile_enable(False, dtype)
    want = dict(zip(("setup", "qkv_finish", "attn", "attn_combine", "commit"), launches))
    for name, p in prof.items():
        assert p["launches"] == want.get(name, 0), name
        assert (p["ms"] > 0) == (p["launches"] > 0) and np.isfinite(p["ms"]) and p["ms"] < 1e3, (name, p)
    step()  # and none when it is off
    torch.cuda.synchronize()
    assert all(p["launches"] == 0 for p in B.profile_read(dtype).values())
