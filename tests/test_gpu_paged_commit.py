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
