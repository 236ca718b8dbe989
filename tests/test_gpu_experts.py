"""The layer of experts on the GPU against 64 bits: choice, shares and outputs."""
import pytest

torch = pytest.importorskip("torch")

import scaled_util as U
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOTH = pytest.mark.parametrize("dtype", ["bf16", "fp16"])
FORMS = pytest.mark.parametrize("scaled", [False, True])


def _randn(dims, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(dims, generator=g) * size).to(U.TYPES[dtype]).to(DEV)


def make(n, d, ff, top_k, dtype, scaled, renormalise=True, seed=0, size=1.0, down=1.0):
    router = _randn((n, d), dtype, 1000 + seed, 1.5 * d ** -0.5)
    experts = [tuple(_randn(dims, dtype, 10 * e + i + 7777 * seed, (down if i == 2 else size) * dims[1] ** -0.5) for i, dims in enumerate([(ff, d), (ff, d), (d, ff)])) for e in range(n)]
    layer = B.ExpertLayer(router, iter(experts), top_k, scaled=scaled, renormalise=renormalise)
    held = [tuple(U.blocks(w, True) if scaled else w.cpu().double() for w in e) for e in experts]
    return layer, router, held


def check(layer, router, held, x, got, rows=None):
    y, chosen, share = got
    want, weight = U.choose(x, router, layer.top_k, layer.renormalise)
    value, error = U.experts(x, held, want, weight)
    bound = U.rounded(value, error, x.dtype)
    keep = slice(None) if rows is None else rows
    assert torch.equal(chosen.cpu().long()[keep], want[keep])
    U.close(share[keep], weight[keep], (weight * 2.0 ** -22 + 2.0 ** -126)[keep], "share")
    U.close(y[keep], value[keep], bound[keep], "y")


# experts, d_model, d_ff, top_k, rows
SHAPES = [(1, 64, 32, 1, 1), (4, 128, 96, 1, 3), (8, 64, 160, 2, 16), (5, 192, 128, 5, 17), (16, 256, 64, 4, 33), (3, 512, 416, 2, 47), (64, 128, 32, 6, 64),
          (2, 320, 288, 1, 80), (512, 64, 32, 16, 80), (130, 64, 64, 8, 79), (8, 1024, 1408, 2, 9), (40, 64, 32, 3, 1), (4, 4096, 256, 2, 5), (6, 64, 4352, 2, 7),
          (32, 64, 64, 16, 17), (33, 128, 32, 16, 31), (17, 192, 32, 3, 33), (2, 64, 128, 1, 80), (3, 64, 96, 3, 80),
          (6, 1024, 96, 3, 9), (2, 320, 1120, 1, 2), (40, 512, 64, 1, 12), (5, 2048, 64, 4, 30), (12, 1536, 64, 4, 50), (4, 4160, 64, 2, 60),
          (4, 2048, 416, 2, 64), (5, 1600, 1120, 2, 40)]


@BOTH
@FORMS
@pytest.mark.parametrize("n,d,ff,top_k,rows", SHAPES)
def test_layers(n, d, ff, top_k, rows, scaled, dtype):
    for renormalise in (True, False):
        layer, router, held = make(n, d, ff, top_k, dtype, scaled, renormalise)
        x = _randn((rows, d), dtype, rows + n)
        got = layer.run(x)
        check(layer, router, held, x, got)
        again = layer.run(x)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


@BOTH
@FORMS
@pytest.mark.parametrize("n,rows", [(6, 15), (6, 16), (6, 33), (6, 80), (100, 17), (100, 49), (200, 80)])
def test_every_row_on_the_same_experts(n, rows, scaled, dtype):
    """One expert has all the rows, and experts have none; with fewer choices than experts and with more."""
    layer, router, held = make(n, 128, 96, 2, dtype, scaled)
    x = _randn((rows, 128), dtype, 3, 0.01) + _randn((1, 128), dtype, 4)
    got = layer.run(x)
    check(layer, router, held, x, got)
    assert len(got[1].unique()) < 6


@BOTH
@FORMS
@pytest.mark.parametrize("n", [8, 33, 90])
def test_rows_that_are_left_out(n, scaled, dtype):
    layer, router, held = make(n, 128, 160, 2, dtype, scaled)
    rows = 40
    x = _randn((rows, 128), dtype, 3)
    position = torch.arange(rows, dtype=torch.int32, device=DEV)
    out_rows = [0, 5, 17, 18, 19, 20, 21, 22, 23, 24, 25, 26, 27, 28, 29, 30, 31, 38, 39]
    position[out_rows] = -1
    x[out_rows] = float("nan")
    keep = [r for r in range(rows) if r not in out_rows]
    y = torch.full_like(x, 7.0)
    chosen, share = torch.full((rows, 2), 9, dtype=torch.int32, device=DEV), torch.full((rows, 2), 3.0, device=DEV)
    got = layer.run(x, y, position=position, chosen=chosen, share=share)
    one = B.ExpertLayer(router, [tuple(w.to(x.dtype).to(DEV) for w in e) for e in held], 1, scaled=scaled)  # one choice a row: another way out
    y1 = one.run(x, torch.full_like(x, 7.0), position=position)[0]
    assert bool((y1[out_rows] == 7).all()) and bool(torch.isfinite(y1[keep]).all()) and not bool((y1[keep] == 7).all(1).any())
    clean = x.clone()
    clean[out_rows] = 0.0
    check(layer, router, held, clean, got, keep)
    assert bool((y[out_rows] == 7).all()) and bool((chosen[out_rows] == 9).all()) and bool((share[out_rows] == 3).all())
    alone = layer.run(x[keep].contiguous())
    assert torch.equal(alone[1], chosen[keep]) and torch.equal(alone[2], share[keep])
    position[:] = -1
    y2 = layer.run(x, torch.full_like(x, 7.0), position=position)[0]
    assert bool((y2 == 7).all())


@BOTH
def test_equal_logits_go_to_the_lowest_experts(dtype):
    layer, router, held = make(70, 64, 32, 3, dtype, False)
    same = torch.zeros_like(router)
    same[11], same[40], same[5], same[69] = 1.0, 1.0, 1.0, 1.0
    experts = [tuple(w.to(U.TYPES[dtype]).to(DEV) for w in e) for e in held]
    layer = B.ExpertLayer(same, experts, 3)
    x = torch.full((2, 64), 0.5, dtype=U.TYPES[dtype], device=DEV)
    x[1] = -0.5
    _, chosen, share = layer.run(x)
    assert chosen.tolist() == [[5, 11, 40], [0, 1, 2]]
    assert torch.equal(share, torch.full_like(share, 1.0 / 3.0))


@BOTH
@FORMS
def test_a_row_of_nan_or_infinities_leaves_the_others_alone(scaled, dtype):
    layer, router, held = make(8, 128, 96, 2, dtype, scaled)
    x = _randn((20, 128), dtype, 3)
    want = layer.run(x)
    bad = x.clone()
    bad[4, 7], bad[17, 100], bad[18] = float("nan"), float("inf"), float("-inf")
    y, chosen, share = layer.run(bad)
    keep = [r for r in range(20) if r not in (4, 17, 18)]
    assert torch.equal(y[keep], want[0][keep]) and torch.equal(chosen[keep], want[1][keep])
    assert bool(torch.isnan(y[[4, 17, 18]]).any(1).all())
    assert chosen[4].tolist() == [0, 1] and bool(((chosen >= 0) & (chosen < 8)).all())


@FORMS
@pytest.mark.parametrize("size,factor,down", [(3.0, 300.0, 1e-3), (0.05, 0.02, 2e4)])
def test_hidden_values_outside_fp16(size, factor, down, scaled):
    """What lies between the two products keeps fp32's range in the fp16 build too: beyond 65504, and far below what fp16 resolves."""
    layer, router, held = make(4, 64, 64, 2, "fp16", scaled, size=size, down=down)
    x = _randn((9, 64), "fp16", 3, factor)
    hidden = max(float(((x.cpu().double() @ g.T) * (x.cpu().double() @ u.T)).abs().max()) for g, u, _ in held)
    assert hidden > 2 * 65504 or hidden < 2.0 ** -14
    check(layer, router, held, x, layer.run(x))


@BOTH
@FORMS
def test_rows_apart_in_place_and_between(scaled, dtype):
    layer, router, held = make(8, 128, 96, 2, dtype, scaled)
    x = _randn((21, 128), dtype, 3)
    want = layer.run(x)[0]
    wide = torch.full((21, 512), 5.0, dtype=x.dtype, device=DEV)
    wide[:, 128:256] = x
    layer.run(wide[:, 128:256], wide[:, 264:392])
    assert torch.equal(wide[:, 264:392], want) and bool((wide[:, 392:] == 5).all()) and bool((wide[:, 256:264] == 5).all())
    layer.run(wide[:, 128:256], wide[:, 128:256])
    assert torch.equal(wide[:, 128:256], want) and bool((wide[:, :128] == 5).all())


def test_no_rows():
    layer, _, _ = make(2, 64, 32, 1, "bf16", True)
    assert layer.run(torch.ones((0, 64), dtype=torch.bfloat16, device=DEV))[0].shape == (0, 64)


@BOTH
@FORMS
@pytest.mark.parametrize("rows", [2, 40])
def test_captured_and_replayed_beside_eager_calls(rows, scaled, dtype):
    layer, router, held = make(16, 128, 160, 4, dtype, scaled)
    x, y = _randn((rows, 128), dtype, 1), torch.zeros((rows, 128), dtype=U.TYPES[dtype], device=DEV)
    layer.run(x, y)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(layer.run(x, y.clone()))
    for seed in range(4):
        fresh = _randn((rows, 128), dtype, 10 + seed)
        x.copy_(fresh)
        for g in graphs:
            g.replay()
        eager = layer.run(fresh)
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_two_streams_at_once():
    layer, router, held = make(16, 256, 416, 4, "bf16", True)
    xs = [_randn((30, 256), "bf16", s) for s in range(2)]
    want = [layer.run(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(layer.run(xs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for g in got[i] for a, b in zip(g, want[i]))


@BOTH
@FORMS
def test_a_mlp_and_a_head_held_in_8_bits(scaled, dtype):
    """A step's tail as a target with experts runs it: the layer of experts on the rows of a padded step, the residual, the LM head's fp32 logits."""
    rows, d, vocab = 9, 256, 1003
    layer, router, held = make(8, d, 352, 2, dtype, scaled)
    head_w = _randn((vocab, d), dtype, 5, d ** -0.5)
    head = B.ScaledMatrix(head_w)
    position = torch.tensor([10, 11, 12, 13, 11, 12, 13, -1, -1], dtype=torch.int32, device=DEV)
    x = _randn((rows, d), dtype, 3)
    y, chosen, _ = layer.run(x, position=position)
    assert bool((y[7:] == 0).all())
    check(layer, router, held, x, (y, chosen, _), list(range(7)))
    x2 = x + y
    logits = head.product(x2, fp32=True)
    U.close(logits, *U.product(x2, U.blocks(head_w, True), torch.float32, False), "logits")
    best = (U.blocks(x2, False) @ U.blocks(head_w, True).T).argmax(1)
    assert torch.equal(logits.argmax(1).cpu(), best)


# experts, top_k -> launches of the router (one for small ones), of the down product (and the sum over a row's experts)
@pytest.mark.parametrize("n,top_k,router_launches,down_launches", [(4, 2, 1, 2), (32, 1, 1, 1), (33, 2, 2, 2)])
@BOTH
def test_timer_sees_the_launches(dtype, n, top_k, router_launches, down_launches):
    layer, _, _ = make(n, 64, 32, top_k, dtype, False)
    x = _randn((5, 64), dtype, 1)
    layer.run(x)
    torch.cuda.synchronize()
    B.profile_enable(True, dtype)
    try:
        layer.run(x)
        assert B.profile_dropped(dtype) == 0
        prof = B.profile_read(dtype)
    finally:
        B.profile_enable(False, dtype)
    want = {"moe_router": router_launches, "moe_gate_up": 1, "moe_down": down_launches}
    assert all(p["launches"] == want.get(name, 0) for name, p in prof.items())


def test_the_binding_refuses():
    router = _randn((4, 64), "bf16", 1)
    one = tuple(_randn(dims, "bf16", 2) for dims in [(32, 64), (32, 64), (64, 32)])
    for experts in ([one] * 3, [one] * 5, [], [tuple(w.half() for w in one)] * 4, [(one[0], one[1], one[0])] * 4):
        with pytest.raises(ValueError):
            B.ExpertLayer(router, experts, 2)
    for top in (0, 5):
        with pytest.raises(ValueError, match="top_k"):
            B.ExpertLayer(router, [one] * 4, top)
    layer = B.ExpertLayer(router, [one] * 4, 2)
    x = _randn((5, 64), "bf16", 3)
    i32 = dict(dtype=torch.int32, device=DEV)
    for kw in ({"x": x.half()}, {"x": x[:, :32]}, {"out": x[:4]}, {"out": x.half()}, {"position": torch.zeros(4, **i32)}, {"position": torch.zeros(5, device=DEV)},
               {"chosen": torch.zeros((5, 3), **i32)}, {"share": torch.zeros((5, 2), dtype=torch.float64, device=DEV)}, {"out": x[:1].expand(5, 64)}):
        with pytest.raises(ValueError):
            layer.run(**{"x": x, **kw})
    with pytest.raises(B.DuoError):
        layer.run(_randn((81, 64), "bf16", 3))
