"""Handles of 8-bit matrices and of layers of experts that are made on one stream and used on others, without a synchronization of the program's own."""
import pytest

torch = pytest.importorskip("torch")

from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = pytest.mark.parametrize("kind", ["matrix", "layer", "layer in 8 bits"])


def _randn(dims, seed, size=1.0):
    return (torch.randn(dims, generator=torch.Generator().manual_seed(seed)) * size).to(torch.bfloat16).to(DEV)


def _sources(kind):
    if kind == "matrix":
        return [_randn((1000, 2048), 1)]
    return [_randn((6, 256), 1)] + [_randn(dims, 2 + i, 0.1) for i, dims in enumerate([(416, 256), (416, 256), (256, 416)])]


def _handle(kind, sources):
    if kind == "matrix":
        return B.ScaledMatrix(sources[0])
    return B.ExpertLayer(sources[0], [tuple(sources[1:])] * 6, 2, scaled="8 bits" in kind)


def _use(handle, x):
    return handle.product(x) if isinstance(handle, B.ScaledMatrix) else handle.run(x)[0]


def _rows(kind):
    return _randn((9, 2048 if kind == "matrix" else 256), 7)


@pytest.fixture(scope="module")
def busy():
    """Some 20 ms of work for the current stream."""
    a = torch.ones((8192, 8192), dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(a)
    torch.matmul(a, a, out=out)
    torch.cuda.synchronize()

    def enqueue():
        for _ in range(24):
            torch.matmul(a, a, out=out)
    return enqueue


@KINDS
def test_a_handle_is_ready_when_its_constructor_returns(kind, busy):
    """Whatever its stream still had to do in front of the packing."""
    sources, side = _sources(kind), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
        handle = _handle(kind, sources)
    assert side.query()
    del handle


@KINDS
def test_used_at_once_on_another_stream(kind, busy):
    sources, x = _sources(kind), _rows(kind)
    want = _use(_handle(kind, sources), x)
    made, used = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(made):
        busy()
        handle = _handle(kind, sources)
    with torch.cuda.stream(used):
        got = _use(handle, x)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@KINDS
def test_captured_at_once_on_another_stream(kind, busy):
    sources, x = _sources(kind), _rows(kind)
    want = _use(_handle(kind, sources), x)
    made = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(made):
        busy()
        handle = _handle(kind, sources)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = _use(handle, x)
    for _ in range(3):
        got.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@KINDS
def test_made_while_its_stream_is_captured(kind):
    """The packing is part of the graph, and so is what the handle is used for there."""
    sources, x = _sources(kind), _rows(kind)
    want = _use(_handle(kind, sources), x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        handle = _handle(kind, sources)
        got = _use(handle, x)
    for _ in range(3):
        got.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@KINDS
@pytest.mark.parametrize("captured", [False, True])
def test_dropped_while_calls_are_on_their_way(kind, captured, busy):
    """The memory of a handle is not handed out while a call on another stream than the handle's own still reads it, also where a captured call
    was the first one there."""
    sources, x = _sources(kind), _rows(kind)
    handle = _handle(kind, sources)
    want = _use(handle, x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    if captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            _use(handle, x)
    held = [(t.data_ptr(), t.numel() * t.element_size()) for t in ([handle.packed] if kind == "matrix" else [handle._packed, handle._router])]
    with torch.cuda.stream(side):
        busy()
        got = _use(handle, x)
    del handle
    others = [torch.full((n,), 0x38, dtype=torch.uint8, device=DEV) for _, n in held for _ in range(3)]
    assert not side.query()  # what follows was asked for while the call was on its way
    assert all(o.data_ptr() + o.numel() <= p or p + n <= o.data_ptr() for o in others for p, n in held)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_streams_are_recorded_once():
    handle, x, side = _handle("layer", _sources("layer")), _rows("layer"), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        first = _use(handle, x)
        known = set(handle._streams)
        again = _use(handle, x)
    torch.cuda.synchronize()
    assert handle._streams == known and len(known) == 2
    assert torch.equal(first, again)
