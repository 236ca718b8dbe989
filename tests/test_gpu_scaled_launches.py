"""Products on 8-bit matrices through every kernel that sizes can choose for up to 80 rows, and with scales and sizes near the ends of their ranges."""
import pytest

torch = pytest.importorskip("torch")

import scaled_util as U
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOTH = pytest.mark.parametrize("dtype", ["bf16", "fp16"])
OUTPUTS = pytest.mark.parametrize("fp32", [True, False])


def _randn(dims, dtype, seed, size=1.0):
    x = torch.randn(dims, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * size
    return x.to(U.TYPES[dtype])


def _wanted(x, held, dtype, eight_bit):
    if held.device.type == "cpu":
        return U.product(x, held, dtype, eight_bit)
    assert not eight_bit
    xv = U.blocks(x, False).to(DEV)  # a matrix of tens of thousands of outputs: in 64 bits on the GPU
    value, error = xv @ held.T, xv.abs() @ held.abs().T * U.sum_steps(x.shape[1])
    return value.cpu(), U.rounded(value, error, dtype).cpu()


def _compare(m, x, fp32, held):
    """The product into the middle of a larger buffer, against 64 bits; what lies around it stays.  held: on either device."""
    rows, left, many = x.shape[0], 16, x.shape[0] > B.DUO_MAX_ROWS and not fp32
    width = left + (m.N + 7) // 8 * 8 + 16
    out = torch.full((rows, width), 7.0, dtype=torch.float32 if fp32 else x.dtype, device=DEV)
    got = m.product(x, out[:, left:left + m.N])
    U.close(got, *_wanted(x, held, got.dtype, many), "product")
    assert bool((out[:, :left] == 7).all()) and bool((out[:, left + m.N:] == 7).all())
    assert torch.equal(got, m.product(x, fp32=fp32))


# rows, N, K -> row tiles, bands of 16 outputs a workgroup, its waves, blocks of columns on their way.  K is such that a wave has more blocks than that.
DIRECT = [  # every workgroup brings the rows to e4m3
    (1, 4090, 2208, "1 1 8 2"), (16, 4099, 2208, "1 2 8 2"), (9, 12290, 1184, "1 4 8 1"), (3, 16500, 2208, "1 2 8 2"), (16, 70001, 2208, "1 2 8 2"),
    (17, 4001, 2016, "2 1 8 1"), (32, 6003, 2048, "2 2 8 1"), (20, 12301, 2016, "2 4 4 2"), (31, 20005, 736, "2 4 4 1"), (18, 66001, 736, "2 4 4 1")]
READY = [  # a launch in front of the product does
    (17, 4095, 2208, "2 1 8 2"), (32, 4113, 2208, "2 2 8 2"), (25, 9003, 2208, "2 4 4 2"), (20, 22016, 2208, "2 2 4 2"), (30, 65535, 2112, "2 2 4 2"), (19, 66002, 2112, "2 4 4 2"),
    (33, 4091, 2208, "3 1 8 2"), (47, 5007, 2208, "3 2 8 2"), (48, 12290, 1184, "3 4 4 2"), (34, 22017, 1184, "3 2 4 2"), (40, 40001, 672, "3 4 2 2"), (33, 66003, 416, "3 4 1 2"),
    (49, 4080, 2208, "4 1 8 2"), (64, 8191, 2208, "4 2 8 2"), (63, 12291, 1184, "4 4 4 2"), (50, 24575, 1184, "4 2 4 2"), (60, 40003, 672, "4 4 2 2"), (64, 70005, 416, "4 4 1 2"),
    (65, 4084, 2208, "5 1 8 2"), (80, 5001, 2208, "5 2 8 2"), (79, 16383, 1184, "5 4 4 2"), (66, 17001, 1184, "5 2 4 2"), (80, 40002, 672, "5 4 2 2"), (75, 65537, 416, "5 4 1 2")]


@BOTH
@pytest.mark.parametrize("rows,N,K,kernel", DIRECT + READY)
def test_every_kernel_of_few_rows(rows, N, K, kernel, dtype):
    assert (rows + 15) // 16 == int(kernel[0])
    m = B.ScaledMatrix(_randn((N, K), dtype, N + K, K ** -0.5))
    x, held = _randn((rows, K), dtype, rows), m.values().double()  # (held values have tests of their own)
    for fp32 in (True, False):
        _compare(m, x, fp32, held)


@OUTPUTS
@pytest.mark.parametrize("rows", [2, 40, 100])
@pytest.mark.parametrize("of_rows,of_matrix", [(118, -105), (-105, 118), (60, -60), (-110, 100)])
def test_scales_near_their_ends(of_rows, of_matrix, rows, fp32):
    """Blocks with scales from 2^-110 to 2^116, whose products lie in the range of the outputs; a block of the other kind beside each."""
    first = (torch.arange(256, device=DEV) < 128)
    x = _randn((rows, 256), "bf16", 1) * torch.where(first, 2.0 ** of_rows, 2.0 ** of_matrix).to(torch.bfloat16)
    w = _randn((200, 256), "bf16", 2) * torch.where(first, 2.0 ** of_matrix, 2.0 ** of_rows).to(torch.bfloat16)
    m = B.ScaledMatrix(w)
    held = U.blocks(w, True)
    scales = m.packed[2 * 2 * 16384:][:4].cpu().int() - 127
    assert int(scales.min()) <= max(min(of_rows, of_matrix) - 5, -110) and int(scales.max()) >= max(of_rows, of_matrix) - 8
    _compare(m, x, fp32, held)


@OUTPUTS
@pytest.mark.parametrize("rows", [1, 17, 80, 100])
def test_the_most_columns(rows, fp32):
    w = _randn((130, B.SCALED_MAX_K), "bf16", 3, 2.0 ** -8)
    _compare(B.ScaledMatrix(w), _randn((rows, B.SCALED_MAX_K), "bf16", 4), fp32, U.blocks(w, True))


@OUTPUTS
@pytest.mark.parametrize("rows,distance", [(3, 2 ** 31 - 8), (20, 2 ** 28), (70, 2 ** 26), (100, 2 ** 25)])
def test_rows_far_apart(rows, distance, fp32):
    """Offsets of rows beyond 32 bits, in the inputs and in the outputs."""
    N, K = 203, 2208
    m = B.ScaledMatrix(_randn((N, K), "bf16", 5, 2.0 ** -5))
    x = _randn((rows, K), "bf16", 6)
    far = torch.empty((rows - 1) * distance + K, dtype=torch.bfloat16, device=DEV).as_strided((rows, K), (distance, 1))
    far.copy_(x)
    out = torch.empty((rows - 1) * distance + N, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV).as_strided((rows, N), (distance, 1))
    assert torch.equal(m.product(far, out), m.product(x, fp32=fp32))


@pytest.mark.parametrize("rows", [3, 40, 100])
def test_a_matrix_beyond_4_GiB(rows):
    """As many outputs as there can be; the first and the last of them against 64 bits."""
    N, K = B.SCALED_MAX_N, 4160
    w = torch.empty((N, K), dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(8))
    m = B.ScaledMatrix(w)
    assert m.packed.numel() > 1 << 32
    ends = [(0, 256), (N - 256, N)]
    held = [U.blocks(w[a:b], True) for a, b in ends]
    del w
    x = _randn((rows, K), "bf16", 9)
    got = m.product(x)
    for (a, b), h in zip(ends, held):
        U.close(got[:, a:b], *U.product(x, h, got.dtype, rows > B.DUO_MAX_ROWS), f"outputs {a} to {b}")


def test_as_many_rows_as_there_can_be():
    """More than 4 GiB of outputs; the first and the last rows against 64 bits."""
    rows, N, K = B.SCALED_MAX_ROWS, 16400, 32
    w, x = _randn((N, K), "fp16", 1), _randn((rows, K), "fp16", 2)
    got = B.ScaledMatrix(w).product(x)
    held = U.blocks(w, True)
    for a, b in ((0, 200), (rows // 2 - 100, rows // 2 + 100), (rows - 200, rows)):
        U.close(got[a:b], *U.product(x[a:b], held, got.dtype, True), f"rows {a} to {b}")


@OUTPUTS
@pytest.mark.parametrize("rows,N,K", [(9, 150, 96), (20, 150, 224), (40, 150, 352), (90, 150, 96), (94, 65, 4448)])
def test_what_lies_around_the_rows_does_not_matter(rows, N, K, fp32):
    """NaN between the rows and behind the last one, columns that end inside a block."""
    w, x = _randn((N, K), "bf16", 1, K ** -0.5), _randn((rows, K), "bf16", 2)
    around = torch.full((rows, K + 72), float("nan"), dtype=torch.bfloat16, device=DEV)
    around[:, 8:8 + K] = x
    m = B.ScaledMatrix(w)
    _compare(m, x, fp32, U.blocks(w, True))
    assert torch.equal(m.product(around[:, 8:8 + K], fp32=fp32), m.product(x, fp32=fp32))


@BOTH
@pytest.mark.parametrize("rows,N,K", [(20, 150, 384), (40, 150, 384), (94, 150, 4448)])
def test_infinities_and_nan_stay_in_their_row_and_their_column(rows, N, K, dtype):
    """Where a launch of its own brings the rows to e4m3, and where the columns are split over workgroups."""
    x, w = _randn((rows, K), dtype, 1), _randn((N, K), dtype, 2, K ** -0.5)
    x[1, 200], x[3, 5], x[rows - 1, K - 1] = float("inf"), float("nan"), float("-inf")
    w[140, 300], w[7, 0] = float("-inf"), float("nan")
    m, held = B.ScaledMatrix(w), U.blocks(w, True)
    for fp32 in (True, False):
        got = m.product(x, fp32=fp32)
        want, bound = U.product(x, held, got.dtype, rows > B.DUO_MAX_ROWS and not fp32)
        bad = torch.zeros((rows, N), dtype=torch.bool)
        bad[[1, 3, rows - 1]] = bad[:, [7, 140]] = True
        assert torch.equal(torch.isnan(got).cpu(), bad)
        U.close(got.cpu()[~bad], want[~bad], bound[~bad])
