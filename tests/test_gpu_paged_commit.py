"""Commit records of every kind: which branch they may name, and records that never leave the device."""
import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("record", [(-2, 0, 9, 0), (-2, 3, 9, 0), (-7, 0, -1, 0), (-2 ** 31, 1, 9, 0), (3, 1, 9, 0), (2 ** 31 - 1, 1, 9, 0), (1, -1, 9, 0)])
def test_a_record_that_names_no_branch_commits_nothing(record):
    """-1 alone says that no branch was accepted; whatever else is no branch of the request is reported, and its neighbours are committed."""
    requests = [(30, 1, 3, 5), (12, 1, 3, 5), (40, 1, 3, 5)]
    cache, lines = U.make(requests, 4, 2, 64, "bf16", 32, layers=2)
    cache.plan()
    assert cache.status.item() == 0
    keys, values = cache.key_pages.clone(), cache.value_pages.clone()
    cache.commit(torch.tensor([(-1, 0, 9, 0), record, (0, 4, 9, 0)], dtype=torch.int32, device=DEV))
    assert cache.status.item() == B.PAGE_BAD_RECORD
    assert cache.cached.tolist() == [31, 12, 45]
    assert torch.equal(keys, cache.key_pages) and torch.equal(values, cache.value_pages)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_records_stay_on_the_device(dtype):
    """Every request's sampler writes its record where the commit reads it, at once (duo_result.commit points into the array) or by a copy on the device
    (NoAllocSampler.commit); the host looks at nothing in between."""
    import ctypes as C
    requests, vocab, L = [(30, 1, 3, 5), (0, 50, 0, 0), (63, 1, 2, 9), (12, 0, 4, 3), (31, 1, 1, 2)], 300, 2
    hq, hkv, D, page = 4, 2, 64, 32
    lib = B.load(dtype)
    g = torch.Generator(device=DEV).manual_seed(4)
    samplers = [B.NoAllocSampler(8, DEV) for _ in requests]
    draws = []
    for cached, trunk, n, k in requests:
        draws.append(None if n * k == 0 else (
            torch.randn((trunk + n * k, vocab), generator=g, device=DEV), torch.randn(vocab, generator=g, device=DEV),
            torch.randint(0, vocab, (n, k), generator=g, device=DEV).int(), torch.softmax(torch.randn((n, k, vocab), generator=g, device=DEV), -1),
            torch.rand((n, k + 1), generator=g, device=DEV) * 0.4))
    outcomes = []
    for way in ("in place", "copied"):
        cache, lines = U.make(requests, hq, hkv, D, dtype, page, layers=L)
        cache.plan()
        keys, values = cache.key_pages.clone(), cache.value_pages.clone()
        records = torch.full((len(requests), 4), -9, dtype=torch.int32, device=DEV)  # a request without branches has no record
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        keep = []
        torch.cuda.synchronize()
        for r, ((cached, trunk, n, k), draw) in enumerate(zip(requests, draws)):
            if draw is None:
                continue
            logits, root, tokens, probs, uniforms = draw
            if way == "copied":
                assert samplers[r].run(*draw, has_root=trunk > 0, prefix_len=cached, dtype=dtype) == 0
                records[r].copy_(samplers[r].commit)
                continue
            need = C.c_size_t()
            assert lib.duo_sample_workspace_bytes(vocab, n, k, C.byref(need)) == 0
            ws, ints = torch.empty(need.value, dtype=torch.uint8, device=DEV), torch.zeros(2 * n, dtype=torch.int32, device=DEV)
            keep.append((ws, ints))
            call = B.Call(n, k, 1.0, 0, 0 if trunk else -1, cached, 0.0)
            result = B.Result(ints.data_ptr(), ints[n:].data_ptr(), records[r].data_ptr(), status.data_ptr(), None)
            assert lib.duo_spec_sample(logits.data_ptr(), root.data_ptr(), vocab, tokens.data_ptr(), probs.data_ptr(), uniforms.data_ptr(), C.byref(call),
                                       C.byref(result), ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == 0
        cache.commit(records)
        assert cache.status.item() == 0 and status.item() == 0
        got = records.tolist()
        outcomes.append(got)
        ik, iv = U.offsets(D, page, "k").to(DEV), U.offsets(D, page, "v").to(DEV)
        after = []
        for r, (cached, trunk, n, k) in enumerate(requests):
            branch, a = got[r][:2] if n * k else (-1, 0)
            after.append(cached + trunk + a)
            assert n * k == 0 or got[r][3] == after[-1]  # the sampler's own new length
            for j in range(a if branch > 0 else 0):
                s, d = cached + trunk + branch * k + j, cached + trunk + j
                for pool, idx in ((keys, ik), (values, iv)):
                    pool[:, lines[r][d // page], :, idx[d % page]] = pool[:, lines[r][s // page], :, idx[s % page]]
        assert cache.cached.tolist() == after
        assert torch.equal(keys, cache.key_pages) and torch.equal(values, cache.value_pages)
    assert outcomes[0] == outcomes[1] and any(x[0] > 0 and x[1] > 0 for x in outcomes[0])
