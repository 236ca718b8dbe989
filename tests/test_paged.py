"""The paged-cache calls without a GPU: refusals, and that whatever the lengths are, a step's schedule fits the workspace."""
import ctypes as C
import functools
import os
import random
import subprocess
import tempfile

import pytest

from paper_2503_00784_amd import binding as B
from paper_2503_00784_amd import inputs

HERE = os.path.dirname(os.path.abspath(__file__))
TILE_ROWS = 128


@functools.lru_cache(maxsize=None)
def rules():
    with tempfile.TemporaryDirectory() as d:
        so = os.path.join(d, "page_rules.so")
        subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "page_rules.cpp"), "-o", so],
                       check=True)
        return C.CDLL(so)


def _layout(requests, max_rows, max_new, max_blocks, hq, hkv, D):
    out = (C.c_longlong * 13)()
    rules().layout(requests, max_rows, max_new, max_blocks, hq, hkv, D, out)
    names = ("stream_items", "tile_items", "stream_parts", "tile_parts", "merges", "stream_rows", "info", "stream", "tile", "merge", "part_stream", "part_tile", "total")
    return dict(zip(names, out))


def _cut(requests, max_new, max_blocks, hq, hkv):
    cached, rows = ((C.c_int * len(requests))(*[r[i] for r in requests]) for i in range(2))
    out = (C.c_int * 6)()
    rules().cut(len(requests), cached, rows, max_new, max_blocks, hq, hkv, out)
    return dict(zip(("stream_items", "tile_items", "stream_parts", "tile_parts", "merges", "covered"), out))


def _fits(requests, hq, hkv, D, max_rows=None, max_new=None, max_slots=None):
    total = sum(r[1] for r in requests)
    max_rows = max(1, total) if max_rows is None else max_rows
    max_new = max(1, max(r[1] for r in requests)) if max_new is None else max_new
    max_slots = max(32, max(r[0] + r[1] for r in requests)) if max_slots is None else max_slots
    max_blocks = (max_slots + 31) // 32
    lay, cut = _layout(len(requests), max_rows, max_new, max_blocks, hq, hkv, D), _cut(requests, max_new, max_blocks, hq, hkv)
    for name in ("stream_items", "tile_items", "stream_parts", "tile_parts", "merges"):
        assert cut[name] <= lay[name], (name, cut[name], lay[name])
    assert cut["covered"] == 1
    group = hq // hkv
    for _, rows in requests:
        if 0 < rows * group <= 64:
            assert rows * group <= lay["stream_rows"]
    assert lay["part_tile"] - lay["part_stream"] >= lay["stream_parts"] * hkv * lay["stream_rows"] * (D + 4) * 4
    assert lay["total"] - lay["part_tile"] >= lay["tile_parts"] * hkv * TILE_ROWS * (D + 4) * 4
    return cut, lay


@pytest.mark.parametrize("seed", range(40))
def test_the_schedule_fits(seed):
    rng = random.Random(seed)
    for _ in range(25):
        hkv = rng.choice([1, 2, 3, 4, 7, 8, 12, 28, 32, 40, 128, 512])
        hq = hkv * rng.choice([g for g in (1, 2, 3, 4, 7, 8, 16, 128) if g * hkv <= 512])
        long = rng.choice([40, 1000, 30000, 200000])
        count = rng.choice([1, 2, 5, 40, 300])
        requests = [(rng.randint(0, long), rng.choice([0, 1, 1, 2, rng.randint(1, 33), rng.randint(1, 1500)])) for _ in range(count)]
        _fits(requests, hq, hkv, rng.choice([64, 128]))


def test_the_schedule_fits_at_the_limits():
    _fits([(B.PAGE_MAX_SLOTS - 1, 1)], 8, 1, 128)
    _fits([(B.PAGE_MAX_SLOTS - 1, 1)] * 4096, 8, 8, 128)
    _fits([(B.PAGE_MAX_SLOTS - 64, 64)] * 4096, 512, 512, 64)
    _fits([(0, B.PAGE_MAX_ROWS)], 512, 1, 64)
    _fits([(B.PAGE_MAX_SLOTS - B.PAGE_MAX_ROWS, B.PAGE_MAX_ROWS)], 64, 64, 128)
    # exactly as many blocks as ranges of equal length, and one more
    for hkv in (1, 28, 12, 7):
        for blocks in (8, 9, 16, 17, 1024 // hkv * 8, 1024 // hkv * 8 + 1):
            _fits([(32 * blocks - 1, 1)], hkv, hkv, 64)
            _fits([(32 * blocks - 1, 1)] * 3, hkv, hkv, 64)


def test_short_steps_are_not_cut():
    cut, _ = _fits([(200, 1)] * 4, 32, 8, 128)
    assert cut["stream_parts"] == 0 and cut["merges"] == 0 and cut["stream_items"] == 4
    cut, _ = _fits([(131000, 1)], 32, 8, 128)
    assert cut["stream_parts"] > 64 and cut["merges"] == 4


# --------------------------------------------------------------------------- refusals: every call made here is refused, nothing is enqueued
A = 0x1000
CALLS = ("plan", "append", "attention", "commit")
ROWS, OUT = (A, 512, A, 128, A, 128, A + 0x100000, 512), (A, 512, A + 0x100000, 512)


def _cfg(hq=8, hkv=2, D=64, layers=2):
    return B.make_config(inputs.ModelShape(layers, 64 * hq, hq, hkv, D, 64, 1000), 32)


def _refused(code, calls, cfg, cache, batch, tables=None, to=None, layer=0, rows=ROWS, out=OUT, scale=0.0, ws=A, nbytes=1 << 40, table=A, records=A,
             cached_out=A):
    """Makes the named calls; each has to return `code`, which is not 0."""
    assert code < 0
    lib = B.load()
    ref = lambda x: None if x is None else C.byref(x)
    tables = B.PageTablesC(A, A, A, A) if tables is None else tables
    for name in calls:
        if name == "plan":
            got = lib.duo_page_plan(ref(cfg), ref(cache), ref(tables), ref(tables if to is None else to), ref(batch), ws, nbytes, None)
        elif name == "append":
            got = lib.duo_page_append(ref(cfg), ref(cache), ref(batch), layer, *rows, None)
        elif name == "attention":
            got = lib.duo_page_attention(ref(cfg), ref(cache), table, ref(batch), layer, *out, scale, ws, nbytes, None)
        else:
            got = lib.duo_page_commit(ref(cfg), ref(cache), table, ref(batch), records, cached_out, ws, nbytes, None)
        assert got == code, name


def _cache(**kw):
    f = dict(k=A, v=A, n_pages=10, page_slots=64, max_pages=4)
    f.update(kw)
    return B.PageCacheC(f["k"], f["v"], f["n_pages"], f["page_slots"], f["max_pages"])


def _batch(n_requests=3, max_rows=40, max_new=20, **kw):
    f = {n: A for n in ("cached", "trunk", "n", "k", "row_start", "position", "slot", "status")}
    f.update(kw)
    return B.PageBatchC(*f.values(), n_requests, max_rows, max_new)


def _size_code(cfg, cache, batch):
    out = C.c_size_t()
    return B.load().duo_page_workspace_bytes(C.byref(cfg), C.byref(cache), C.byref(batch), C.byref(out))


@pytest.mark.parametrize("bad", [dict(n_pages=0), dict(page_slots=0), dict(page_slots=16), dict(page_slots=48), dict(page_slots=2048), dict(max_pages=0),
                                 dict(n_pages=1 << 26), dict(max_pages=1 << 18), dict(page_slots=-64), dict(n_pages=-1), dict(max_pages=-1)])
def test_geometry_is_refused(bad):
    cfg, cache, batch = _cfg(), _cache(**bad), _batch()
    assert _size_code(cfg, cache, batch) == -2
    _refused(-2, CALLS, cfg, cache, batch)


@pytest.mark.parametrize("bad", [dict(n_requests=0), dict(n_requests=4097), dict(max_rows=0), dict(max_rows=262145), dict(max_new=0), dict(max_new=41), dict(n_requests=-1),
                                 dict(max_new=-3)])
def test_maxima_are_refused(bad):
    cfg, cache, batch = _cfg(), _cache(), _batch(**bad)
    assert _size_code(cfg, cache, batch) == -2
    _refused(-2, CALLS, cfg, cache, batch)


def test_models_are_refused():
    for cfg in (_cfg(D=96), _cfg(hq=7, hkv=2)):
        assert _size_code(cfg, _cache(), _batch()) == -2
        _refused(-2, CALLS, cfg, _cache(), _batch())
    lib, out = B.load(), C.c_size_t()
    assert lib.duo_page_workspace_bytes(None, C.byref(_cache()), C.byref(_batch()), C.byref(out)) == -1
    assert lib.duo_page_workspace_bytes(C.byref(_cfg()), None, C.byref(_batch()), C.byref(out)) == -1
    assert lib.duo_page_workspace_bytes(C.byref(_cfg()), C.byref(_cache()), None, C.byref(out)) == -1
    assert lib.duo_page_workspace_bytes(C.byref(_cfg()), C.byref(_cache()), C.byref(_batch()), None) == -1
    _refused(-1, CALLS, None, _cache(), _batch())
    _refused(-1, CALLS, _cfg(), None, _batch())
    _refused(-1, CALLS, _cfg(), _cache(), None)


def test_pointers_are_refused():
    cfg, cache, batch = _cfg(), _cache(), _batch()
    for name in ("cached", "trunk", "n", "k", "row_start", "position", "slot", "status"):
        for bad, code in ((None, -1), (A + 2, -4)):
            calls = ["plan"] + ["append"] * (name in ("position", "slot", "status")) + ["attention"] * (name == "status") + ["commit"] * (name in ("status", "cached"))
            _refused(code, calls, cfg, cache, _batch(**{name: bad}))
    for field in range(4):
        for bad, code in ((None, -1), (A + 2, -4)):
            t = [A, A + 64, A + 128, A + 192]
            t[field] = bad
            _refused(code, ["plan"], cfg, cache, batch, tables=B.PageTablesC(*t))
            _refused(code, ["plan"], cfg, cache, batch, to=B.PageTablesC(*t))
    _refused(-8, ["plan"], cfg, cache, batch, to=B.PageTablesC(A, A, A, A + 4))  # in place in part
    for bad, code in ((None, -1), (A + 8, -4)):
        _refused(code, ["plan", "attention", "commit"], cfg, cache, batch, ws=bad)
        for pool in ("k", "v"):
            _refused(code, ["append", "attention", "commit"], cfg, _cache(**{pool: bad}), batch)
    need = C.c_size_t()
    B.load().duo_page_workspace_bytes(C.byref(cfg), C.byref(cache), C.byref(batch), C.byref(need))
    _refused(-5, ["plan", "attention", "commit"], cfg, cache, batch, nbytes=need.value - 1)
    for bad, code in ((None, -1), (A + 2, -4)):
        _refused(code, ["attention", "commit"], cfg, cache, batch, table=bad)
        _refused(code, ["commit"], cfg, cache, batch, records=bad)
        _refused(code, ["commit"], cfg, cache, batch, cached_out=bad)


def test_rows_are_refused():
    cfg, cache, batch = _cfg(), _cache(), _batch()
    for i in range(0, 8, 2):
        for at, bad, code in ((i, None, -1), (i, A + 8, -4), (i + 1, ROWS[i + 1] + 4, -4), (i + 1, ROWS[i + 1] - 8, -2), (i + 1, -512, -2)):
            rows = list(ROWS)
            rows[at] = bad
            _refused(code, ["append"], cfg, cache, batch, rows=rows)
    _refused(-8, ["append"], cfg, cache, batch, rows=(A, 512, A, 128, A, 128, A, 520))  # in place with other rows
    for i in (0, 2):
        for at, bad, code in ((i, None, -1), (i, A + 8, -4), (i + 1, 516, -4), (i + 1, 504, -2)):
            out = list(OUT)
            out[at] = bad
            _refused(code, ["attention"], cfg, cache, batch, out=out)
    _refused(-8, ["attention"], cfg, cache, batch, out=(A, 512, A, 512))
    for layer in (-1, 2):
        _refused(-8, ["append", "attention"], cfg, cache, batch, layer=layer)
    for scale in (-1.0, float("nan"), float("inf")):
        _refused(-8, ["attention"], cfg, cache, batch, scale=scale)


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    shape = inputs.ModelShape(2, 512, 8, 2, 64, 64, 1000)
    make = lambda **kw: B.PagedCache(shape, **{**dict(n_pages=10, max_requests=3, max_pages=4, max_rows=40, max_new=20, device="cpu"), **kw})
    for bad in (dict(page_slots=40), dict(max_requests=0), dict(max_rows=0), dict(max_new=50), dict(n_pages=0), dict(max_pages=0)):
        with pytest.raises(B.DuoError):
            make(**bad)
    c = make()
    q, kv = torch.zeros((40, 8, 64), dtype=torch.bfloat16), torch.zeros((40, 128), dtype=torch.bfloat16)
    for bad in (q[:39], q.half(), q.float(), q.transpose(1, 2), q[:, :4], torch.zeros((40, 64, 8), dtype=torch.bfloat16), torch.zeros((40, 8, 128), dtype=torch.bfloat16)[..., ::2],
                torch.zeros((40, 16, 64), dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            c.append(0, bad, kv, kv)
        with pytest.raises(ValueError):
            c.attention(0, bad, q)
        with pytest.raises(ValueError):
            c.attention(0, q, bad)
    with pytest.raises(ValueError):
        c.append(0, q, kv, kv[:, :64])
    with pytest.raises(ValueError):
        c.append(0, q, kv, kv, torch.zeros((1, 8, 64), dtype=torch.bfloat16).expand(40, 8, 64))
    records = torch.zeros((3, 4), dtype=torch.int32)
    for bad in (records.long(), records[:2], torch.zeros((3, 8), dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            c.commit(bad)
    for bad in (torch.zeros(2, dtype=torch.int32), torch.zeros(3), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            c.commit(records, bad)
    for n in (0, 4, -1):
        with pytest.raises(ValueError):
            c.plan(n)
    with pytest.raises(ValueError):
        c.plan(source=B.PageTables(torch.zeros((3, 5), dtype=torch.int32), *c.tables.tensors()[1:]))
    with pytest.raises(ValueError):
        c.set_requests([1] * 4, [0] * 4, [0] * 4)
    for bad in (torch.zeros((3, 4)), torch.zeros((3, 8), dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            B.PageTables(bad, *c.tables.tensors()[1:])
    with pytest.raises(ValueError):
        c.tables = B.PageTables.empty(2, 4, 10, "cpu")
    for name in ("cached", "key_pages", "status", "workspace"):
        with pytest.raises(AttributeError):
            setattr(c, name, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(AttributeError):
        c.tables.held = torch.zeros(3, dtype=torch.int32)


def test_a_cache_on_the_cpu_runs_nothing():
    torch = pytest.importorskip("torch")
    shape = inputs.ModelShape(2, 512, 8, 2, 64, 64, 1000)
    c = B.PagedCache(shape, n_pages=10, max_requests=3, max_pages=4, max_rows=40, max_new=20, device="cpu")
    q, kv = torch.zeros((40, 8, 64), dtype=torch.bfloat16), torch.zeros((40, 128), dtype=torch.bfloat16)
    for call in (c.plan, lambda: c.append(0, q, kv, kv), lambda: c.attention(0, q), lambda: c.commit(torch.zeros((3, 4), dtype=torch.int32))):
        with pytest.raises(ValueError, match="on cpu"):
            call()
