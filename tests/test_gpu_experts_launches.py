"""Layers of experts through every kernel that their sizes can choose, with one choice a row and with more; experts with many more rows than the mean;
the largest sizes."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_experts import DEV, _randn, check, make
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "fp16"])
FORMS = pytest.mark.parametrize("scaled", [False, True])

# experts, d_model, d_ff, top_k, rows -> of the down product: row tiles, bands of 16 outputs a workgroup, its waves
ONE = [(12, 1536, 544, 1, 16, "1 4 2"), (4, 2048, 1312, 1, 9, "1 2 4"), (4, 512, 1184, 1, 9, "1 1 8"),
       (4, 4160, 672, 1, 60, "2 4 4"), (2, 4096, 1184, 1, 40, "2 2 8"), (2, 1024, 1184, 1, 40, "2 1 8"),
       (2, 6208, 672, 1, 70, "3 4 4"), (2, 4096, 1184, 1, 70, "3 2 8"), (2, 1088, 1184, 1, 79, "3 1 8")]
MORE = [(12, 1536, 544, 2, 16, "1 4 2"), (4, 2048, 1312, 2, 9, "1 2 4"), (4, 512, 1184, 2, 9, "1 1 8"),
        (4, 3136, 672, 2, 40, "2 4 4"), (4, 2048, 1184, 2, 40, "2 2 8"), (4, 512, 1184, 2, 40, "2 1 8"),
        (3, 4160, 672, 2, 50, "3 4 4"), (3, 2048, 1184, 2, 50, "3 2 8"), (3, 576, 1184, 2, 80, "3 1 8")]


def test_the_shapes_are_of_the_tiles_they_name():
    for n, d, ff, top_k, rows, kernel in ONE + MORE:
        each = rows * top_k // n
        assert (1 if each <= 12 or rows <= 16 else 2 if each <= 28 else 3) == int(kernel[0])


@BOTH
@FORMS
@pytest.mark.parametrize("n,d,ff,top_k,rows,kernel", ONE + MORE)
def test_every_kernel(n, d, ff, top_k, rows, kernel, scaled, dtype):
    layer, router, held = make(n, d, ff, top_k, dtype, scaled)
    wide = torch.full((rows, d + 64), 5.0, dtype=router.dtype, device=DEV)
    x = _randn((rows, d), dtype, rows)
    got = layer.run(x, wide[:, 32:32 + d])
    check(layer, router, held, x, got)
    assert bool((wide[:, :32] == 5).all()) and bool((wide[:, 32 + d:] == 5).all())
    assert all(torch.equal(a, b) for a, b in zip(got, layer.run(x)))


# experts, d_model, d_ff, rows: most rows on the same experts, several times as many as the row tiles of the kernels hold
@BOTH
@FORMS
@pytest.mark.parametrize("top_k", [1, 2])
@pytest.mark.parametrize("n,d,ff,rows", [(20, 4160, 96, 80), (14, 1024, 416, 80), (20, 64, 1184, 79), (5, 4160, 96, 80), (5, 1024, 1184, 80), (5, 64, 1184, 77), (90, 4160, 32, 80)])
def test_most_rows_on_the_same_experts(n, d, ff, rows, top_k, scaled, dtype):
    layer, router, held = make(n, d, ff, top_k, dtype, scaled)
    x = _randn((rows, d), dtype, 3, 0.01) + _randn((1, d), dtype, 4)
    x[::8] = _randn((len(range(0, rows, 8)), d), dtype, 5)  # and some elsewhere
    got = layer.run(x)
    check(layer, router, held, x, got)
    assert int(torch.bincount(got[1].flatten().long()).max()) > rows // 2


@FORMS
@pytest.mark.parametrize("n,d,ff,top_k,rows", [(2, 8192, 96, 2, 3), (3, 8192, 96, 1, 80), (2, 64, B.SCALED_MAX_K, 1, 3), (2, 64, B.SCALED_MAX_K, 2, 33)])
def test_the_largest_sizes(n, d, ff, top_k, rows, scaled):
    layer, router, held = make(n, d, ff, top_k, "bf16", scaled)
    x = _randn((rows, d), "bf16", rows)
    check(layer, router, held, x, layer.run(x))


@FORMS
@pytest.mark.parametrize("top_k", [1, 2])
def test_rows_as_far_apart_as_they_can_be(top_k, scaled):
    n, d, rows, distance = 6, 192, 80, 1 << 23
    layer, _, _ = make(n, d, 160, top_k, "bf16", scaled)
    x = _randn((rows, d), "bf16", 6)
    far, out = (torch.empty((rows - 1) * distance + d, dtype=torch.bfloat16, device=DEV).as_strided((rows, d), (distance, 1)) for _ in range(2))
    far.copy_(x)
    want, got = layer.run(x), layer.run(far, out)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
