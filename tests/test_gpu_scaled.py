"""Matrices in 8 bits with block scales and products with them, on the GPU, against 64 bits."""
import pytest

torch = pytest.importorskip("torch")

import scaled_util as U
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOTH = pytest.mark.parametrize("dtype", ["bf16", "fp16"])


def _randn(dims, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(dims, generator=g) * size
    x = torch.where(torch.rand(dims, generator=g) < 0.01, x * 30, x)
    return x.to(U.TYPES[dtype]).to(DEV)


@BOTH
@pytest.mark.parametrize("N,K", [(1, 32), (16, 128), (17, 96), (128, 160), (130, 128), (257, 1056), (515, 416)])
def test_held_values(N, K, dtype):
    w = _randn((N, K), dtype, N + K) * torch.logspace(-2, 2, N, device=DEV)[:, None].to(U.TYPES[dtype])
    assert torch.equal(B.ScaledMatrix(w).values().cpu().double(), U.blocks(w, True))


@BOTH
def test_every_value_of_the_type_in_blocks_of_every_size(dtype):
    """All finite 16-bit patterns, a block of each largest value: the rounding and the scale are those of the definition, bit for bit.  (bf16 magnitudes
    from 1.9375 * 2^127 on, half way between e4m3's 240 * 2^120 and 256 * 2^120, round to 2^128, which is infinite in fp32.)"""
    pattern = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(U.TYPES[dtype])
    finite = pattern[torch.isfinite(pattern)].float().abs().sort(stable=True).values.to(U.TYPES[dtype])  # neighbours share a block
    finite = torch.where(torch.arange(len(finite)) % 2 == 0, finite, -finite)
    w = torch.nn.functional.pad(finite, (0, -len(finite) % 256)).reshape(-1, 256).to(DEV)
    assert torch.equal(B.ScaledMatrix(w).values().cpu(), U.blocks(w, True).float())
    x = finite[torch.randperm(len(finite), generator=torch.Generator().manual_seed(3))]                  # and large ones beside small ones
    x = torch.nn.functional.pad(x, (0, -len(x) % 256)).reshape(-1, 256).to(DEV)
    assert torch.equal(B.ScaledMatrix(x).values().cpu(), U.blocks(x, True).float())


@BOTH
@pytest.mark.parametrize("rows", [1, 16, 37, 80, 81, 300])
@pytest.mark.parametrize("fp32", [True, False])
def test_rows_times_the_identity_are_the_rows_in_8_bits(rows, fp32, dtype):
    """Each output is one product: what the rows became, without a rounding in fp32 and with the type's own in 16 bits."""
    K = 288
    x = _randn((rows, K), dtype, rows) * torch.logspace(-3, 2, K, device=DEV).to(U.TYPES[dtype])
    x[0, :128] = 0.0
    eye = B.ScaledMatrix(torch.eye(K, device=DEV, dtype=U.TYPES[dtype]))
    want = U.blocks(x, False)
    got = eye.product(x, fp32=fp32)
    assert torch.equal(got.cpu().double(), want if fp32 else want.to(U.TYPES[dtype]).double())


SHAPES = [(1, 64, 128), (1, 4096, 4096), (2, 17, 32), (5, 1, 96), (8, 130, 1056), (15, 515, 416), (16, 256, 2048), (17, 100, 352), (33, 1031, 1408), (48, 48, 5120),
          (49, 300, 160), (64, 4099, 512), (79, 128, 11008), (80, 640, 608), (81, 640, 608), (100, 33, 96), (128, 128, 128), (129, 1000, 1408), (257, 515, 4096),
          (600, 4099, 288), (1023, 2050, 1056),
          (100, 9000, 160), (500, 4096, 416), (999, 12290, 160), (2000, 4096, 288), (999, 5120, 416), (1500, 8200, 96), (90, 200, 4096), (128, 40000, 96),
          (26, 96, 14784), (17, 4096, 4096), (30, 9000, 2080), (32, 20000, 96), (18, 70000, 32), (25, 8000, 2112), (40, 70000, 32), (66, 20000, 64), (50, 25000, 64),
          # every size of block, of 16-bit and of fp32 outputs
          (521, 16820, 96), (399, 16512, 160), (393, 12508, 96), (258, 16706, 96), (403, 11415, 160), (259, 13643, 96), (260, 16312, 96), (129, 16565, 288),
          (82, 16487, 416), (81, 8299, 416), (92, 109, 416),
          # columns split over two, four and eight workgroups
          (8221, 65, 5344), (4112, 65, 3456), (1037, 142, 4064), (1035, 133, 2560), (533, 133, 4224), (142, 4510, 5280), (87, 69, 2176), (94, 65, 4448),
          (2192, 141, 2848), (2170, 73, 6016), (99, 73, 1728), (120, 1699, 12224)]


@BOTH
@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("rows,N,K", SHAPES)
def test_products(rows, N, K, fp32, dtype):
    x, w = _randn((rows, K), dtype, 7 * rows + N), _randn((N, K), dtype, N + 3 * K, K ** -0.5)
    m = B.ScaledMatrix(w)
    got = m.product(x, fp32=fp32)
    assert got.shape == (rows, N) and got.dtype == (torch.float32 if fp32 else U.TYPES[dtype])
    U.close(got, *U.product(x, U.blocks(w, True), got.dtype, rows > B.DUO_MAX_ROWS and not fp32), "product")
    assert torch.equal(got, m.product(x, fp32=fp32))  # and the same bits again


@BOTH
@pytest.mark.parametrize("rows,K", [(3, 224), (33, 224), (130, 224), (90, 4448)])
@pytest.mark.parametrize("fp32", [True, False])
def test_rows_apart_and_what_lies_between_them(rows, K, fp32, dtype):
    N = 203
    t = torch.float32 if fp32 else U.TYPES[dtype]
    wide = _randn((rows, 3 * K), dtype, 5)
    x = wide[:, K:2 * K]
    w = _randn((N, K), dtype, 6)
    out = torch.full((rows, 256), 7.0, dtype=t, device=DEV)
    m = B.ScaledMatrix(w)
    got = m.product(x, out[:, 8:8 + N])
    assert got.data_ptr() == out[:, 8:].data_ptr()
    assert torch.equal(got, m.product(x.contiguous(), fp32=fp32))
    assert bool((out[:, :8] == 7).all()) and bool((out[:, 8 + N:] == 7).all())


@BOTH
@pytest.mark.parametrize("rows", [4, 90])
def test_infinities_and_nan_stay_in_their_row_and_their_column(rows, dtype):
    N, K = 150, 384
    x, w = _randn((rows, K), dtype, 1), _randn((N, K), dtype, 2)
    x[1, 200], x[3, 5] = float("inf"), float("nan")
    w[140, 300], w[7, 0] = float("-inf"), float("nan")
    for fp32 in (True, False):
        got = B.ScaledMatrix(w).product(x, fp32=fp32)
        want, bound = U.product(x, U.blocks(w, True), got.dtype, rows > 80 and not fp32)
        nan = torch.isnan(got).cpu()
        assert bool(nan[[1, 3]].all()) and bool(nan[:, [7, 140]].all())
        keep_r, keep_n = [r for r in range(rows) if r not in (1, 3)], [n for n in range(N) if n not in (7, 140)]
        U.close(got.cpu()[keep_r][:, keep_n], want[keep_r][:, keep_n], bound[keep_r][:, keep_n])


@pytest.mark.parametrize("rows", [2, 100])
def test_large_and_small_values(rows):
    """Blocks near both ends of bf16's range, and rows of zeros."""
    K, N = 256, 64
    x, w = _randn((rows, K), "bf16", 1), _randn((N, K), "bf16", 2)
    x = x * torch.where(torch.arange(rows, device=DEV) % 2 == 0, 1e30, 1e-30)[:, None].to(torch.bfloat16)
    x[rows - 1] = 0.0
    w[:, 128:] *= 1e-4
    m = B.ScaledMatrix(w)
    got = m.product(x, fp32=True)
    U.close(got, *U.product(x, U.blocks(w, True), torch.float32, False))
    assert bool((got[rows - 1] == 0).all())


def test_no_rows():
    m = B.ScaledMatrix(torch.ones((16, 32), dtype=torch.bfloat16, device=DEV))
    assert m.product(torch.ones((0, 32), dtype=torch.bfloat16, device=DEV)).shape == (0, 16)


@BOTH
@pytest.mark.parametrize("rows,K", [(9, 512), (200, 512), (100, 4096)])
def test_captured_and_replayed_beside_eager_calls(rows, K, dtype):
    N = 300
    w = _randn((N, K), dtype, 2)
    m = B.ScaledMatrix(w)
    x, out = _randn((rows, K), dtype, 1), torch.zeros((rows, 304), dtype=U.TYPES[dtype], device=DEV)[:, :N]
    m.product(x, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.product(x, out)
    for seed in range(4):
        fresh = _randn((rows, K), dtype, 10 + seed)
        x.copy_(fresh)
        g.replay()
        eager = m.product(fresh)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("rows", [9, 200])
def test_two_streams_at_once(rows):
    N, K = 1000, 2048
    m = B.ScaledMatrix(_randn((N, K), "bf16", 2))
    xs = [_randn((rows, K), "bf16", s) for s in range(2)]
    want = [m.product(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(m.product(xs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])


@BOTH
def test_timer_sees_the_launches(dtype):
    m = B.ScaledMatrix(_randn((100, 256), dtype, 2))
    few, many = _randn((16, 256), dtype, 1), _randn((90, 256), dtype, 1)
    m.product(few), m.product(many)
    torch.cuda.synchronize()
    B.profile_enable(True, dtype)
    try:
        m.product(few)
        first = B.profile_read(dtype)
        m.product(many)
        second = B.profile_read(dtype)
    finally:
        B.profile_enable(False, dtype)
    assert (first["scaled_gemm"]["launches"], second["scaled_gemm"]["launches"]) == (1, 2)
    assert all(p["launches"] == 0 for name, p in {**first, **second}.items() if name != "scaled_gemm")


def test_bytes_lie_where_the_layout_says():
    N, K = 300, 288
    w = _randn((N, K), "bf16", 4)
    held, packed = U.blocks(w, True), B.ScaledMatrix(w).packed.cpu()
    NB, KB = 3, 3
    for n, k in [(0, 0), (15, 127), (16, 64), (129, 130), (299, 287), (200, 191), (77, 15), (78, 16)]:
        byte = ((n // 16) * KB + k // 128) * 2048 + ((k % 128) // 64) * 1024 + ((k % 64) // 16) * 256 + (n % 16) * 16 + k % 16
        scale = packed[NB * KB * 16384 + (n // 128) * KB + k // 128].item() - 127
        assert packed[byte:byte + 1].view(torch.float8_e4m3fn).double().item() * 2.0 ** scale == held[n, k].item()


def test_the_binding_refuses():
    m = B.ScaledMatrix(torch.ones((64, 96), dtype=torch.bfloat16, device=DEV))
    x = torch.ones((4, 96), dtype=torch.bfloat16, device=DEV)
    for bad in (x.half(), x.float(), x[:, :64], x.cpu(), x[0], torch.ones((96, 4), dtype=torch.bfloat16, device=DEV).t()):
        with pytest.raises(ValueError):
            m.product(bad)
    for out in (torch.empty((3, 64), dtype=x.dtype, device=DEV), torch.empty((4, 65), dtype=x.dtype, device=DEV), torch.empty((4, 64), dtype=torch.float16, device=DEV),
                torch.empty((4, 64), dtype=torch.float64, device=DEV), torch.empty((1, 64), dtype=x.dtype, device=DEV).expand(4, 64)):
        with pytest.raises(ValueError):
            m.product(x, out)
    with pytest.raises(B.DuoError):  # rows that are not 16 bytes apart
        m.product(torch.ones((4, 97), dtype=torch.bfloat16, device=DEV)[:, :96])
    with pytest.raises(B.DuoError):  # over its input
        wide = torch.ones((4, 192), dtype=torch.bfloat16, device=DEV)
        m.product(wide[:, :96], wide[:, 96:160])
    with pytest.raises(ValueError, match="multiple of 32"):
        B.ScaledMatrix(torch.ones((64, 40), dtype=torch.bfloat16, device=DEV))
