"""How many entries the per-kernel timer writes: duo_profile_read fills the twelve classes it was published with, whatever was added since."""
import ctypes as C

import pytest

from paper_2503_00784_amd import binding as B

CLASSES, ALL = 12, 16


@pytest.fixture(params=["bf16", "fp16"])
def lib(request):
    return B.load(request.param)


def _arrays(n):
    return (C.c_double * n)(*[7.5] * n), (C.c_int32 * n)(*[-3] * n)


def test_arrays_of_twelve_entries_are_enough(lib):
    ms, launches = _arrays(ALL)
    assert lib.duo_profile_read(ms, launches) == 0
    assert list(ms) == [0.0] * CLASSES + [7.5] * (ALL - CLASSES)
    assert list(launches) == [0] * CLASSES + [-3] * (ALL - CLASSES)


@pytest.mark.parametrize("classes", [1, 12, 13, 16, 20])
def test_as_many_entries_as_are_asked_for(lib, classes):
    ms, launches = _arrays(24)
    assert lib.duo_profile_read_classes(ms, launches, classes) == 0
    assert list(ms) == [0.0] * classes + [7.5] * (24 - classes)
    assert list(launches) == [0] * classes + [-3] * (24 - classes)


def test_refusals(lib):
    ms, launches = _arrays(ALL)
    assert lib.duo_profile_read(None, launches) == lib.duo_profile_read(ms, None) == -1
    assert lib.duo_profile_read_classes(None, launches, ALL) == lib.duo_profile_read_classes(ms, None, ALL) == -1
    assert lib.duo_profile_read_classes(ms, launches, 0) == lib.duo_profile_read_classes(ms, launches, -1) == -8
    assert list(ms) == [7.5] * ALL and list(launches) == [-3] * ALL


def test_the_binding_has_a_name_for_every_class():
    assert len(B.PROF_CLASSES) == ALL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_launches_of_the_classes_behind_are_left_out(dtype):
    """A read of twelve classes with launches of a thirteenth among those recorded: none is counted elsewhere, and the next read starts anew."""
    import torch
    t = torch.float16 if dtype == "fp16" else torch.bfloat16
    lib, m, x = B.load(dtype), B.ScaledMatrix(torch.ones((32, 64), dtype=t, device="cuda:0")), torch.ones((3, 64), dtype=t, device="cuda:0")
    m.product(x)
    torch.cuda.synchronize()
    B.profile_enable(True, dtype)
    try:
        m.product(x)
        ms, launches = _arrays(ALL)
        assert lib.duo_profile_read(ms, launches) == 0
        again = B.profile_read(dtype)
        m.product(x)
        counted = B.profile_read(dtype)
    finally:
        B.profile_enable(False, dtype)
    assert list(ms) == [0.0] * CLASSES + [7.5] * 4 and list(launches) == [0] * CLASSES + [-3] * 4
    assert all(p["launches"] == 0 for p in again.values())
    assert {c: p["launches"] for c, p in counted.items() if p["launches"]} == {"scaled_gemm": 1}
