"""What a refused call of the binding leaves behind: nothing.  Without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2503_00784_amd import binding as B
from paper_2503_00784_amd import inputs


@pytest.fixture
def cache():
    return B.PagedCache(inputs.ModelShape(2, 512, 8, 2, 64, 64, 1000), n_pages=10, max_requests=3, max_pages=4, max_rows=40, max_new=20, device="cpu")


@pytest.mark.parametrize("lists", [([7, 7, 7], [5, 5, 5, 5], [6, 6, 6], None), ([7, 7, 7], [5, 5, 5], [6, 6, 6], [9] * 4), ([7, 7], [5], [6, 6], None),
                                   ([7, 7, 7], [], [6, 6, 6], None), ([7], [5], [6, 6], None), ([7, 7], [5, 5], [6, 6], [9]), ([7, 7, 7], [5, 5, 5], [1 << 40] * 3, None),
                                   ([7, 7, 7], [5, 5, 5], [6, 6, "x"], None)])
def test_requests_are_set_whole_or_not_at_all(cache, lists):
    """Lists of other lengths, or too long, or of other things: no request keeps the branches of one step and the trunk of another."""
    cache.set_requests([1, 2, 3], [4, 0, 1], [2, 0, 3], [30, 31, 32])
    with pytest.raises((ValueError, RuntimeError, TypeError)):
        cache.set_requests(*lists)
    assert [x.tolist() for x in (cache.trunk, cache.n, cache.k, cache.cached)] == [[1, 2, 3], [4, 0, 1], [2, 0, 3], [30, 31, 32]]


def test_requests_that_are_set(cache):
    cache.set_requests([1, 2, 3], [4, 0, 1], [2, 0, 3], [30, 31, 32])
    cache.set_requests((5, 6), iter((0, 2)), [1, 1])  # the first two; what is cached stays
    assert [x.tolist() for x in (cache.trunk, cache.n, cache.k, cache.cached)] == [[5, 6, 3], [0, 2, 1], [1, 1, 3], [30, 31, 32]]
    cache.set_requests([], [], [])
    assert cache.trunk.tolist() == [5, 6, 3]


def test_a_plan_that_is_not_enqueued_leaves_the_one_before(cache):
    """The calls behind it still belong to a step of the requests planned last."""
    with pytest.raises(ValueError, match="on cpu"):
        cache.plan(2)
    with pytest.raises(ValueError, match="on cpu"):
        cache.commit(torch.zeros((3, 4), dtype=torch.int32))
    with pytest.raises(ValueError, match="records"):
        cache.commit(torch.zeros((2, 4), dtype=torch.int32))


@pytest.mark.gpu
def test_a_refused_plan_leaves_the_step_before():
    """Tables that are in place in part are refused; attention and commit of the planned step go on."""
    import paged_util as U
    cache, _ = U.make([(40, 1, 0, 0), (3, 5, 0, 0)], 4, 2, 64, "bf16", 32)
    q = torch.randn((cache.max_rows, 4, 64), device="cuda:0").bfloat16()
    cache.plan()
    want = cache.attention(0, q).clone()
    block_table, *others = cache.tables.tensors()
    with pytest.raises(B.DuoError):
        cache.plan(1, source=B.PageTables(block_table.clone(), *others))
    assert torch.equal(cache.attention(0, q), want) and cache.status.item() == 0
    cache.commit(torch.tensor([[-1, 0, 1, 0]] * 2, dtype=torch.int32, device="cuda:0"))
    assert cache.cached.tolist() == [41, 8] and cache.status.item() == 0


@pytest.mark.gpu
def test_streams_without_the_short_way_to_them(monkeypatch):
    """The public call names the same stream: a step's calls on a stream of their own, in order behind what that stream does before."""
    import paged_util as U

    def outputs():
        cache, _ = U.make([(40, 1, 0, 0), (3, 5, 0, 0)], 4, 2, 64, "bf16", 32)
        q = torch.randn((cache.max_rows, 4, 64), generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0").bfloat16()
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            assert cache._stream_of(0) == stream.cuda_stream
            late = torch.zeros_like(q)
            for _ in range(50):
                late.copy_(q)
            cache.plan()
            out = cache.attention(0, late)
        stream.synchronize()
        assert cache.status.item() == 0
        return out

    want = outputs()
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert torch.equal(outputs(), want)
