"""What the calls on 8-bit matrices and the layer of experts refuse, and the sizes they state; no GPU: nothing is enqueued."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2503_00784_amd import binding as B

A = 0x10000  # addresses that are never followed


@pytest.fixture(scope="module", params=["bf16", "fp16"])
def lib(request):
    return B.load(request.param)


def test_bytes_of_a_matrix(lib):
    assert lib.duo_scaled_bytes(1, 32) == 16384 + 16
    assert lib.duo_scaled_bytes(128, 128) == 16384 + 16
    assert lib.duo_scaled_bytes(129, 4096) == 2 * 32 * 16384 + 64
    assert lib.duo_scaled_bytes(B.SCALED_MAX_N, B.SCALED_MAX_K) == B.SCALED_MAX_N * B.SCALED_MAX_K + 8192 * 512
    for n, k in [(0, 32), (-1, 32), (16, 0), (16, 16), (16, 48), (B.SCALED_MAX_N + 1, 32), (16, B.SCALED_MAX_K + 32), (16, -32)]:
        assert lib.duo_scaled_bytes(n, k) == 0


def test_pack_refuses(lib):
    f = lib.duo_scaled_pack
    assert f(None, 16, 32, A, None) == f(A, 16, 32, None, None) == -1
    assert f(A, 0, 32, A, None) == f(A, 16, 31, A, None) == f(A, 16, 0, A, None) == -2
    assert f(A + 8, 16, 32, A, None) == f(A, 16, 32, A + 4, None) == -4


def test_workspace_of_a_product(lib):
    out = C.c_size_t(7)
    f = lib.duo_scaled_workspace_bytes
    assert f(1, 16, 32, None) == -1
    assert f(0, 16, 32, C.byref(out)) == f(B.SCALED_MAX_ROWS + 1, 16, 32, C.byref(out)) == f(1, 16, 33, C.byref(out)) == f(1, 0, 32, C.byref(out)) == -2
    assert out.value == 7
    assert f(16, 4096, 4096, C.byref(out)) == 0 and out.value == 0
    assert f(17, 4096, 4096, C.byref(out)) == 0 and out.value >= 17 * 4096
    assert f(33, 4096, 4096, C.byref(out)) == 0 and out.value >= 33 * 4096
    assert f(81, 4096, 4096, C.byref(out)) == 0 and out.value >= 81 * 4096


def _gemm(lib, x=A, xs=256, w=A << 8, y=A << 16, ys=64, fp32=0, rows=4, n=64, k=256, ws=None, nbytes=0):
    return lib.duo_scaled_gemm(x, xs, w, y, ys, fp32, rows, n, k, ws, nbytes, None)


def test_product_refuses(lib):
    assert _gemm(lib, x=None) == _gemm(lib, w=None) == _gemm(lib, y=None) == -1
    for bad in ({"rows": 0}, {"rows": B.SCALED_MAX_ROWS + 1}, {"k": 0}, {"k": 255}, {"n": 0}, {"xs": 248}, {"ys": 56}, {"xs": -256}, {"xs": 2 ** 31 + 8}, {"ys": 2 ** 40}):
        assert _gemm(lib, **bad) == -2, bad
    for bad in ({"x": A + 8}, {"y": (A << 16) + 8}, {"w": (A << 8) + 1}, {"xs": 257}, {"ys": 68}, {"fp32": 1, "ys": 66}):
        assert _gemm(lib, **bad) == -4, bad
    assert _gemm(lib, fp32=2) == _gemm(lib, fp32=-1) == -8


def test_product_refuses_outputs_over_its_inputs(lib):
    x_end = A + 2 * (3 * 256 + 256)
    assert _gemm(lib, y=A) == _gemm(lib, y=x_end - 16) == _gemm(lib, y=A - 16) == -8
    w = A << 8
    w_end = w + lib.duo_scaled_bytes(64, 256)
    assert _gemm(lib, y=w) == _gemm(lib, y=w_end - 16) == _gemm(lib, y=w - 16) == -8


def test_many_rows_need_a_workspace(lib):
    need = C.c_size_t()
    assert lib.duo_scaled_workspace_bytes(100, 64, 256, C.byref(need)) == 0
    assert _gemm(lib, rows=100) == -1
    assert _gemm(lib, rows=100, ws=A << 4, nbytes=need.value - 1) == -5
    assert _gemm(lib, rows=100, ws=(A << 4) + 8, nbytes=need.value) == -4


def _cfg(**change):
    return B.MoeConfigC(**{**dict(d_model=128, d_ff=96, n_experts=8, top_k=2, scaled=0, renormalise=1), **change})


BAD_SHAPES = [{"d_model": 0}, {"d_model": 96}, {"d_model": 8256}, {"d_ff": 0}, {"d_ff": 48}, {"d_ff": B.SCALED_MAX_K + 32}, {"n_experts": 0}, {"n_experts": 513},
              {"top_k": 0}, {"top_k": 9}, {"top_k": 17, "n_experts": 100}, {"d_model": -64}]


def test_sizes_of_a_layer(lib):
    out = C.c_size_t(7)
    assert lib.duo_moe_expert_bytes(C.byref(_cfg())) == 3 * 2 * 128 * 96
    assert lib.duo_moe_expert_bytes(C.byref(_cfg(scaled=1))) == 2 * lib.duo_scaled_bytes(96, 128) + lib.duo_scaled_bytes(128, 96)
    assert lib.duo_moe_expert_bytes(None) == 0
    assert lib.duo_moe_workspace_bytes(C.byref(_cfg()), 4, None) == lib.duo_moe_workspace_bytes(None, 4, C.byref(out)) == -1
    for rows in (0, -1, 81):
        assert lib.duo_moe_workspace_bytes(C.byref(_cfg()), rows, C.byref(out)) == -2
    for bad in BAD_SHAPES:
        assert lib.duo_moe_expert_bytes(C.byref(_cfg(**bad))) == 0, bad
        assert lib.duo_moe_workspace_bytes(C.byref(_cfg(**bad)), 4, C.byref(out)) == -2, bad
    for bad in ({"scaled": 2}, {"renormalise": -1}):
        assert lib.duo_moe_workspace_bytes(C.byref(_cfg(**bad)), 4, C.byref(out)) == -8
    assert out.value == 7
    assert lib.duo_moe_workspace_bytes(C.byref(_cfg()), 80, C.byref(out)) == 0 and out.value > 80 * 2 * 96 * 4


def test_packing_an_expert_refuses(lib):
    def f(cfg=_cfg(), g=A, u=A, d=A, e=0, dst=A):
        return lib.duo_moe_pack(C.byref(cfg), g, u, d, e, dst, None)
    assert lib.duo_moe_pack(None, A, A, A, 0, A, None) == -1
    assert f(g=None) == f(u=None) == f(d=None) == f(dst=None) == -1
    assert f(e=-1) == f(e=8) == -8
    assert f(g=A + 2) == f(u=A + 2) == f(d=A + 2) == f(dst=A + 8) == -4
    assert f(_cfg(d_model=100)) == -2


def _layer(lib, cfg=None, router=A, experts=A, x=A << 8, xs=128, rows=4, position=None, y=A << 16, ys=128, chosen=None, share=None, ws=A << 4, nbytes=None):
    cfg = cfg or _cfg()
    if nbytes is None:
        out = C.c_size_t()
        lib.duo_moe_workspace_bytes(C.byref(cfg), min(max(rows, 1), 80), C.byref(out))
        nbytes = out.value
    return lib.duo_moe_layer(C.byref(cfg), router, experts, x, xs, rows, position, y, ys, chosen, share, ws, nbytes, None)


def test_layer_refuses(lib):
    for name in ("router", "experts", "x", "y", "ws"):
        assert _layer(lib, **{name: None}) == -1, name
    for rows in (0, -3, 81):
        assert _layer(lib, rows=rows) == -2
    for bad in BAD_SHAPES:
        assert _layer(lib, _cfg(**bad), nbytes=1 << 40) == -2, bad
    for bad in ({"xs": 120}, {"ys": 64}, {"xs": 2 ** 23 + 8}, {"ys": 2 ** 23 + 8}, {"ys": -128}):
        assert _layer(lib, **bad) == -2, bad
    for bad in ({"router": A + 8}, {"experts": A + 4}, {"x": A + 2}, {"y": A + 8}, {"ws": A + 8}, {"xs": 132}, {"ys": 130}, {"position": A + 2}, {"chosen": A + 1},
                {"share": A + 3}):
        assert _layer(lib, **bad) == -4, bad
    assert _layer(lib, _cfg(scaled=3)) == -8
    out = C.c_size_t()
    assert lib.duo_moe_workspace_bytes(C.byref(_cfg()), 4, C.byref(out)) == 0
    assert _layer(lib, nbytes=out.value - 1) == -5


def test_the_binding_refuses_the_cpu_and_other_types():
    with pytest.raises(ValueError, match="GPU"):
        B.ScaledMatrix(torch.zeros((16, 32), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="bfloat16 or torch.float16"):
        B.ScaledMatrix(torch.zeros((16, 32)))
    with pytest.raises(ValueError, match="two dimensions"):
        B.ScaledMatrix(torch.zeros(32, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="GPU"):
        B.ExpertLayer(torch.zeros((4, 64), dtype=torch.float16), [], 1)
    with pytest.raises(ValueError, match="matrix"):
        B.ExpertLayer(torch.zeros(64, dtype=torch.float16), [], 1)
