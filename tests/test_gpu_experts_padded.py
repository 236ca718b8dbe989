"""Layers of experts on padded steps inside a graph, and on more than 4 GiB of experts."""
import pytest

torch = pytest.importorskip("torch")

import scaled_util as U
from test_gpu_experts import DEV, _randn, check, make
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
FORMS = pytest.mark.parametrize("scaled", [False, True])


@FORMS
@pytest.mark.parametrize("n,top_k", [(8, 2), (40, 3), (6, 1)])
def test_rows_left_out_change_from_replay_to_replay(n, top_k, scaled):
    """The positions are read when the graph runs: each replay leaves out the rows that are marked then, and what the call itself makes for them is zeros
    again."""
    rows, d = 24, 128
    layer, router, held = make(n, d, 160, top_k, "bf16", scaled)
    x, position = _randn((rows, d), "bf16", 1), torch.zeros(rows, dtype=torch.int32, device=DEV)
    layer.run(x, position=position)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = layer.run(x, position=position)
    for seed, live in enumerate([24, 5, 0, 17, 24, 1]):
        position.copy_(torch.where(torch.arange(rows) < live, 7, -1).to(torch.int32))
        x.copy_(_randn((rows, d), "bf16", 20 + seed))
        g.replay()
        eager = layer.run(x, position=position)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), live
        assert all(not bool(a[live:].any()) for a in got), live
        check(layer, router, held, x, got, list(range(live)))


@FORMS
def test_experts_beyond_4_GiB(scaled):
    """Rows on the first, a middle and the last expert; the last one's matrices are others than the rest's."""
    n, d, ff = (12, 4096, 16384) if not scaled else (24, 4096, 16384)
    gen = torch.Generator(device=DEV).manual_seed(3)
    both = [[(torch.randn(dims, generator=gen, device=DEV) * dims[1] ** -0.5).bfloat16() for dims in ((ff, d), (ff, d), (d, ff))] for _ in range(2)]
    router = torch.zeros((n, d), dtype=torch.bfloat16, device=DEV)
    router[torch.arange(n), torch.arange(n)] = 1.0
    layer = B.ExpertLayer(router, (both[e == n - 1] for e in range(n)), 1, scaled=scaled)
    assert layer._packed.numel() > 1 << 32
    x = (torch.randn((3, d), generator=gen, device=DEV) * 0.5).bfloat16()
    wanted = [0, n // 2, n - 1]
    x[torch.arange(3), torch.tensor(wanted)] = 9.0
    held = [[m.double().cpu() for m in (b if not scaled else [B.ScaledMatrix(w).values() for w in b])] for b in both]
    y, chosen, share = layer.run(x)
    assert chosen[:, 0].tolist() == wanted and bool((share == 1).all())
    value, error = U.experts(x, [held[e == n - 1] for e in range(n)], chosen.cpu().long(), share.cpu().double())
    U.close(y, value, U.rounded(value, error, y.dtype), "y")


@FORMS
@pytest.mark.parametrize("n,d,ff,top_k,rows", [(6, 192, 96, 2, 9), (6, 64, 32, 1, 9), (2, 320, 160, 2, 40), (2, 192, 224, 1, 80)])
def test_what_lies_around_the_rows_does_not_matter(n, d, ff, top_k, rows, scaled):
    """Sizes that end inside a block of 128 columns, NaN between the rows, behind the last one and in the rows that are left out, the last among them."""
    layer, router, held = make(n, d, ff, top_k, "bf16", scaled)
    x = _randn((rows, d), "bf16", 4)
    around = torch.full((rows, d + 72), float("nan"), dtype=torch.bfloat16, device=DEV)
    around[:, 8:8 + d] = x
    position = torch.arange(rows, dtype=torch.int32, device=DEV)
    position[[1, rows - 2, rows - 1]] = -1
    live = [r for r in range(rows) if r not in (1, rows - 2, rows - 1)]
    around[[1, rows - 2, rows - 1]] = float("nan")
    got = layer.run(around[:, 8:8 + d], position=position)
    check(layer, router, held, x, got, live)
    assert not any(bool(a[[1, rows - 2, rows - 1]].any()) for a in got)
