"""The paged-cache calls against plain 64-bit implementations: plans, appends, attention, commits, and steps of all four."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


# --------------------------------------------------------------------------- plan
def _plan_inputs(R, page, seed, big=300):
    rng = random.Random(seed)
    requests, lines = [], []
    for r in range(R):
        kind = rng.randrange(5)
        if kind == 0:
            requests.append((0, 0, 0, 0))
        elif kind == 1:
            requests.append((0, rng.randint(1, big), 0, 0))
        else:
            requests.append((rng.choice([0, 1, page - 1, page, rng.randint(0, 5 * page)]), rng.randint(0, 2), rng.randint(0, 3), rng.randint(0, 9)))
    need = [-(-(q[0] + U.new_rows(q)) // page) for q in requests]
    held = [max(0, m + rng.randint(-3, 3)) for m in need]
    n_pages = max(sum(need), sum(held)) + rng.randint(0, 5)
    ids = list(range(n_pages))
    rng.shuffle(ids)
    at = 0
    for h in held:
        lines.append(ids[at:at + h])
        at += h
    return requests, lines, ids[at:], n_pages, max(max(need), max(held)) + rng.randint(0, 2)


def _planner(requests, lines, free, n_pages, max_pages, page, pad=4, **kw):
    rows = sum(map(U.new_rows, requests))
    cache = B.PagedCache(U.shape_of(4, 2, 64), n_pages=n_pages, max_requests=len(requests), max_pages=max(1, max_pages), max_rows=rows + pad,
                         max_new=max(1, max(map(U.new_rows, requests))), page_slots=page, **kw)
    U.set_tables(cache, lines, free)
    cache.set_requests([r[1] for r in requests], [r[2] for r in requests], [r[3] for r in requests], [r[0] for r in requests])
    return cache


def _check_plan(cache, want, tables):
    row_start, position, slot, lines, held, stack = want
    R = len(held)
    assert cache.status.item() == 0
    assert cache.row_start[:R + 1].tolist() == row_start
    assert cache.position.tolist() == position
    assert cache.slot.tolist() == slot
    assert tables.held[:R].tolist() == held
    got = tables.block_table.tolist()
    assert [x[:len(y)] for x, y in zip(got, lines)] == lines
    assert tables.free_count.item() == len(stack)
    assert tables.free_pages[:len(stack)].tolist() == stack


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("R,page,seed", [(1, 32, 0), (1, 32, 3), (3, 64, 1), (8, 32, 7), (9, 32, 8), (64, 64, 9), (65, 32, 10), (70, 32, 2), (257, 128, 4), (1024, 32, 11),
                                         (1025, 32, 12), (1100, 32, 5), (4096, 32, 6)])
def test_plan(R, page, seed, in_place):
    requests, lines, free, n_pages, max_pages = _plan_inputs(R, page, seed)
    if sum(map(U.new_rows, requests)) == 0:
        requests[0] = (3, 1, 0, 0)
    want = U.plan(requests, page, (lines, free), sum(map(U.new_rows, requests)) + 4)
    cache = _planner(requests, lines, free, n_pages, max_pages + 12, page)
    if in_place:
        cache.plan()
    else:
        source = B.PageTables(*[t.clone() for t in cache.tables.tensors()])
        before = [t.clone() for t in source.tensors()]
        for t in cache.tables.tensors():
            t.fill_(-7)
        cache.plan(source=source)
        for a, b in zip(before, source.tensors()):
            assert torch.equal(a, b)
    _check_plan(cache, want, cache.tables)
    if not in_place:  # columns and entries beyond are left as they were
        for r, line in enumerate(want[3][:50]):
            assert (cache.tables.block_table[r, len(line):] == -7).all()
        assert (cache.tables.free_pages[len(want[5]):] == -7).all()


def test_a_plan_of_some_requests_leaves_the_others():
    """The first 5 of 12 requests: the others keep their pages."""
    requests, lines, free, n_pages, max_pages = _plan_inputs(12, 32, 21)
    cache = _planner(requests, lines, free, n_pages, max_pages + 12, 32)
    want = U.plan(requests[:5], 32, (lines[:5], free), sum(map(U.new_rows, requests)) + 4)
    cache.plan(5)
    _check_plan(cache, want, cache.tables)
    assert cache.tables.held[5:].tolist() == [len(x) for x in lines[5:]]
    assert [x[:len(y)] for x, y in zip(cache.tables.block_table[5:].tolist(), lines[5:])] == lines[5:]


def test_plan_again_changes_nothing():
    requests, lines, free, n_pages, max_pages = _plan_inputs(40, 32, 9)
    cache = _planner(requests, lines, free, n_pages, max_pages + 12, 32)
    cache.plan()
    first = [t.clone() for t in (*cache.tables.tensors(), cache.slot, cache.position, cache.row_start)]
    cache.plan()
    for a, b in zip(first, (*cache.tables.tensors(), cache.slot, cache.position, cache.row_start)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("what", ["pages", "negative", "too_long", "too_many_rows", "held", "free_count", "huge"])
def test_a_failed_plan_changes_nothing(what, in_place):
    requests = [(40, 1, 2, 3), (0, 50, 0, 0), (10, 1, 0, 0)]
    lines, free = [[5, 2], [], [7]], [0, 1, 3]
    cache = _planner(requests, lines, free, 9, 4, 32)
    cache.plan()
    assert cache.status.item() == 0
    U.set_tables(cache, lines, free)
    status = B.PAGE_BAD_REQUEST
    if what == "pages":
        cache.tables.free_count.fill_(1)
        status = B.PAGE_NO_PAGES
    elif what == "negative":
        cache.trunk[1] = -1
    elif what == "too_long":
        cache.cached[0] = 4 * 32 - 6
    elif what == "too_many_rows":
        cache.trunk[2] = 20
    elif what == "held":
        cache.tables.held[1] = 5
    elif what == "free_count":
        cache.tables.free_count.fill_(10)
    else:
        cache.n[0], cache.k[0] = 1 << 30, 1 << 30
    source = cache.tables
    before = [t.clone() for t in source.tensors()]
    if not in_place:
        cache.tables = B.PageTables(*[torch.full_like(t, -7) for t in before])
    cache.plan(source=source)
    assert cache.status.item() == status
    for a, b in zip(before, source.tensors()):
        assert torch.equal(a, b)
    assert (cache.slot == -1).all() and (cache.position == -1).all() and (cache.row_start == 0).all()
    if not in_place:
        assert torch.equal(cache.tables.held, before[1]) and torch.equal(cache.tables.free_count, before[3])
    # the calls behind it do nothing
    q = torch.randn((cache.max_rows, 4, 64), device=DEV).bfloat16()
    pools = [cache.key_pages.clone(), cache.value_pages.clone()]
    kv = q[:, :2].contiguous()
    out = torch.full_like(q, 3.0)
    cache.append(0, q, kv, kv, torch.empty_like(q))
    cache.attention(0, q, out)
    cached = cache.cached.clone()
    cache.commit(torch.zeros((3, 4), dtype=torch.int32, device=DEV))
    assert torch.equal(pools[0], cache.key_pages) and torch.equal(pools[1], cache.value_pages) and (out == 3.0).all()
    assert torch.equal(cached, cache.cached)


# --------------------------------------------------------------------------- append
@pytest.mark.parametrize("hq,hkv,D,dtype,page,far", [(4, 4, 64, "bf16", 32, 0), (8, 2, 128, "bf16", 64, 5000), (14, 2, 64, "fp16", 128, 131000),
                                                     (3, 1, 128, "fp16", 32, 1000000), (40, 40, 128, "bf16", 256, 77)])
def test_append(hq, hkv, D, dtype, page, far):
    requests = [(far % 97, 1, 3, 5), (0, 45, 0, 0), (31, 2, 0, 0), (0, 0, 0, 0), (64, 0, 1, 9)]
    cache, lines = U.make(requests, hq, hkv, D, dtype, page, layers=2, theta=500000.0)
    cache.plan()
    cache.position[:20] += far  # a caller's own positions
    rows, t = sum(map(U.new_rows, requests)), U.TYPES[dtype]
    qkv = (torch.randn((cache.max_rows, (hq + 2 * hkv) * D + 16), device=DEV) * 1.28).to(t)
    q, k, v = qkv[:, :hq * D], qkv[:, hq * D:(hq + hkv) * D], qkv[:, (hq + hkv) * D:(hq + 2 * hkv) * D]
    pools = [cache.key_pages.clone(), cache.value_pages.clone()]
    out = torch.full((cache.max_rows, hq, D), 7.0, dtype=t, device=DEV)
    cache.append(1, q, k, v, out)
    assert cache.status.item() == 0
    # 64 bits, on the host
    pos = cache.position[:rows].cpu().double()
    angle = pos[:, None] * 500000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turn(x, heads):
        x = x[:rows].cpu().double().reshape(rows, heads, D)
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1), torch.cat([a.abs() + b.abs()] * 2, -1)

    u = torch.finfo(t).eps / 2
    # one rounding of the output; sine and cosine of an angle that fp32 holds to 2 pi 2^-24 of a turn, and fp32 products
    ok = lambda got, want, size: ((got.double() - want).abs() <= u * want.abs() + size * 2.0 ** -20 + 2.0 ** -24).all()
    want, size = turn(q, hq)
    assert ok(out[:rows].cpu(), want, size)
    assert (out[rows:] == 7.0).all()
    slot = cache.slot[:rows].cpu()
    pid, w = slot // page, slot % page
    want, size = turn(k, hkv)
    ik, iv = U.offsets(D, page, "k"), U.offsets(D, page, "v")
    keys, values = cache.key_pages[1].cpu().view(t), cache.value_pages[1].cpu().view(t)
    for h in range(hkv):
        assert ok(keys[pid[:, None], h, ik[w]], want[:, h], size[:, h])
        assert torch.equal(values[pid[:, None], h, iv[w]], v[:rows].cpu().reshape(rows, hkv, D)[:, h])
    # nothing else is touched
    for pool, was, idx in ((cache.key_pages, pools[0], ik), (cache.value_pages, pools[1], iv)):
        assert torch.equal(pool[0], was[0])
        mine, old = pool[1].cpu().clone(), was[1].cpu()
        for h in range(hkv):
            mine[pid[:, None], h, idx[w]] = old[pid[:, None], h, idx[w]]
        assert torch.equal(mine, old)
    # in place
    qc = q.contiguous()
    cache.append(1, qc, k, v)
    assert torch.equal(qc[:rows].view(rows, hq, D), out[:rows])
    assert torch.equal(qc[rows:], q[rows:])


def test_append_of_odd_slots():
    """Rows in any order and page, values with infinities and NaN, slots outside the pool."""
    cache, _ = U.make([(0, 9, 0, 0)], 2, 2, 64, "bf16", 32, spare=4, pad=0)
    cache.plan()
    cache.slot.copy_(torch.tensor([3 * 32 + 7, -1, 31, 5 * 32, 2 * 32 + 8, 2 ** 31 - 1, 0, 3 * 32 + 6, 33], dtype=torch.int32))
    cache.position.copy_(torch.arange(9, dtype=torch.int32))
    x = torch.randn((9, 2, 64), device=DEV).bfloat16()
    x[0, 0, 3], x[2, 1, 0] = math.nan, math.inf
    before = cache.value_pages.clone()
    cache.append(0, x.clone(), x, x, torch.empty_like(x))
    assert cache.status.item() == B.PAGE_BAD_PAGE
    iv = U.offsets(64, 32, "v").to(DEV)
    want = before[0].clone()
    for r, s in enumerate(cache.slot.tolist()):
        if 0 <= s < 5 * 32:
            for h in range(2):
                want[s // 32, h, iv[s % 32]] = x[r, h].view(torch.int16)
    assert torch.equal(cache.value_pages[0], want)


# --------------------------------------------------------------------------- attention
HEADS = {"mha64": (3, 3, 64), "gqa64": (8, 2, 64), "mha128": (2, 2, 128), "gqa128": (8, 2, 128), "odd": (14, 2, 128), "wide": (16, 1, 64), "many": (40, 40, 64)}
STEPS = {
    "one": [(0, 1, 0, 0)],
    "two": [(1, 1, 0, 0)],
    "decode": [(5, 1, 0, 0), (31, 1, 0, 0), (32, 1, 0, 0), (300, 1, 0, 0), (0, 0, 0, 0), (63, 1, 0, 0), (1000, 1, 0, 0)],
    "branches": [(7, 1, 2, 3), (100, 1, 4, 5), (0, 0, 3, 2), (33, 0, 1, 8), (64, 3, 2, 2), (600, 1, 1, 1)],
    "prompt": [(0, 33, 0, 0), (0, 64, 0, 0), (0, 257, 0, 0), (0, 5, 0, 0)],
    "chunk": [(40, 130, 0, 0), (515, 200, 0, 0), (96, 32, 3, 20)],
    "mixed": [(300, 1, 0, 0), (0, 150, 0, 0), (77, 1, 3, 4), (250, 90, 2, 30), (0, 0, 0, 0), (9, 1, 0, 0)],
    "long": [(5000, 1, 0, 0), (3, 1, 0, 0)],
    "long_branches": [(4000, 1, 3, 5)],
    "long_chunk": [(4100, 70, 2, 10)],
}


def _attend(requests, hq, hkv, D, dtype, page, seed=0, layers=1, scale=None, poison=None, q_scale=1.28, **kw):
    cache, lines = U.make(requests, hq, hkv, D, dtype, page, layers=layers, seed=seed, **kw)
    cache.plan()
    assert cache.status.item() == 0
    t = U.TYPES[dtype]
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    wide = (torch.randn((cache.max_rows, hq * D + 24), generator=g, device=DEV) * q_scale).to(t)
    q = wide[:, 8:8 + hq * D]
    if poison:
        poison(cache, lines, q)
    out = torch.full((cache.max_rows, hq * D + 8), 9.0, dtype=t, device=DEV)
    cache.attention(layers - 1, q, out[:, :hq * D], 0.0 if scale is None else scale)
    return cache, lines, q, out


def _compare(requests, cache, lines, q, out, hq, hkv, D, dtype, scale=None, where=None):
    rows = sum(map(U.new_rows, requests))
    t = U.TYPES[dtype]
    keys, values = cache.key_pages[-1].view(t), cache.value_pages[-1].view(t)
    want, mean_abs, size = U.attention(requests, lines, keys, values, q[:rows].reshape(rows, hq, D), hq, hkv, D, scale)
    got = out[:rows, :hq * D].reshape(rows, hq, D).double()
    assert (out[rows:] == 9.0).all() and (out[:, hq * D:] == 9.0).all()
    row0, worst = 0, 0.0
    for r, line in zip(requests, lines):
        new = U.new_rows(r)
        if new == 0:
            continue
        part = slice(row0, row0 + new)
        v_max = float(torch.nan_to_num(values[torch.tensor(line, device=DEV)].float(), 0.0, 0.0, 0.0).abs().max())
        bound = U.attention_bound(want[part], mean_abs[part], size[part], dtype, D, r[0] + new, v_max, new * (hq // hkv) <= 64)
        err = (got[part] - want[part]).abs()
        if where is not None:
            err, bound = err[where[part]], bound[where[part]]
        assert torch.isfinite(err).all(), r
        worst = max(worst, float((err / bound).max()))
        assert (err <= bound).all(), (r, float((err / bound).max()))
        row0 += new
    say("largest error over bound", worst)
    return want, got


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("step", list(STEPS))
def test_attention(step, heads, dtype):
    hq, hkv, D = HEADS[heads]
    say(step, heads, dtype)
    page = {"one": 32, "two": 64, "decode": 32, "branches": 64, "prompt": 128, "chunk": 32, "mixed": 64, "long": 256, "long_branches": 32, "long_chunk": 1024}[step]
    requests = STEPS[step]
    cache, lines, q, out = _attend(requests, hq, hkv, D, dtype, page, layers=2 if step == "mixed" else 1)
    _compare(requests, cache, lines, q, out, hq, hkv, D, dtype)
    assert cache.status.item() == 0


@pytest.mark.parametrize("rows", [1, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 129, 160, 255, 256, 257])
@pytest.mark.parametrize("D,cached", [(64, 0), (64, 701), (128, 95), (128, 1500)])
def test_attention_at_the_sizes_where_the_kernels_change(rows, D, cached):
    """One request of `rows` rows of one head: short ones in one range, long ones cut."""
    dtype = "fp16" if rows % 2 else "bf16"
    requests = [(cached, rows, 0, 0)] if rows % 3 else [(cached, rows - 2 * (rows // 3), 2, rows // 3)]
    say(rows, D, cached, requests)
    cache, lines, q, out = _attend(requests, 1, 1, D, dtype, 32, seed=rows)
    _compare(requests, cache, lines, q, out, 1, 1, D, dtype)


@pytest.mark.parametrize("blocks", [1, 7, 8, 9, 16, 17, 23, 24, 25, 31, 32, 33, 64, 65])
@pytest.mark.parametrize("new", [1, 20, 50, 70])
def test_attention_at_the_lengths_where_ranges_change(blocks, new):
    for total in (32 * blocks, 32 * blocks - 1, 32 * blocks + 1):
        if total < new:
            continue
        requests = [(total - new, new, 0, 0)]
        cache, lines, q, out = _attend(requests, 2, 2, 64, "bf16", 64, seed=blocks)
        _compare(requests, cache, lines, q, out, 2, 2, 64, "bf16")


@pytest.mark.parametrize("new", [1, 5, 20])
@pytest.mark.parametrize("D", [64, 128])
def test_short_requests_beside_a_long_one(new, D):
    """The table has room for long requests: short ones are cut too, in the shortest ranges and one block beyond them."""
    requests = [(2500, 1, 0, 0)] + [(32 * blocks - new + d, new, 0, 0) for blocks in (1, 4, 5, 8, 9, 12, 13, 16, 17) for d in (-1, 0, 1)]
    cache, lines, q, out = _attend(requests, 2, 1, D, "fp16", 64, seed=new)
    _compare(requests, cache, lines, q, out, 2, 1, D, "fp16")


@pytest.mark.parametrize("seed", range(6))
def test_attention_of_random_steps(seed):
    rng = random.Random(seed)
    hq, hkv, D = rng.choice(list(HEADS.values()))
    requests = []
    for _ in range(rng.randint(1, 9)):
        requests.append((rng.choice([0, rng.randint(0, 2500)]), rng.choice([0, 1, 1, rng.randint(1, 300)]), rng.randint(0, 4), rng.randint(0, 20)))
    requests.append((rng.randint(0, 100), 1, 0, 0))
    dtype, page = rng.choice(["bf16", "fp16"]), rng.choice([32, 64, 128, 512])
    say(seed, (hq, hkv, D), dtype, page, requests)
    cache, lines, q, out = _attend(requests, hq, hkv, D, dtype, page, seed=seed)
    _compare(requests, cache, lines, q, out, hq, hkv, D, dtype)


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_attention_scale(scale):
    requests = [(90, 1, 2, 3), (10, 120, 0, 0)]
    cache, lines, q, out = _attend(requests, 4, 2, 64, "bf16", 32, scale=scale)
    _compare(requests, cache, lines, q, out, 4, 2, 64, "bf16", scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("requests,D", [([(20, 1, 3, 4)], 128), ([(0, 1, 0, 0)], 128), ([(70, 60, 2, 25), (5, 1, 0, 0)], 128), ([(3000, 1, 2, 2)], 128),
                                        ([(2500, 80, 0, 0)], 128), ([(40, 3, 4, 6)], 128), ([(1700, 3, 4, 6), (9, 1, 2, 2)], 64), ([(33, 2, 2, 2)], 64),
                                        ([(130, 2, 3, 4)], 64), ([(100, 40, 3, 30), (7, 1, 1, 2)], 64)])
def test_what_is_not_seen_does_not_touch_a_row(requests, D, dtype):
    """Slots behind a request's last hold NaN; one branch (or the last trunk row) brings infinities and NaN in keys and values.  Rows that do not see
    it are as if it were not there, rows that do are what the formula gives."""
    hq, hkv, page = 4, 2, 64
    t = U.TYPES[dtype]

    def poison(cache, lines, q):
        for kind, pool in (("k", cache.key_pages), ("v", cache.value_pages)):
            flat = pool[0].view(t)
            idx = U.offsets(D, page, kind).to(DEV)
            for r, line in zip(requests, lines):
                total = r[0] + U.new_rows(r)
                for s in range(total, len(line) * page):
                    flat[line[s // page], :, idx[s % page]] = math.nan
                if U.new_rows(r) > 1:
                    s = total - 1
                    flat[line[s // page], :, idx[s % page][5]] = math.inf if kind == "v" else math.nan
                    if U.new_rows(r) > 2:
                        flat[line[(s - 1) // page], 1, idx[(s - 1) % page][D - 1]] = math.nan

    cache, lines, q, out = _attend(requests, hq, hkv, D, dtype, page, poison=poison)
    rows = sum(map(U.new_rows, requests))
    clean = torch.ones((rows, hq, D), dtype=torch.bool, device=DEV)
    row0 = 0
    for r in requests:
        new = U.new_rows(r)
        see = U.visible(r)
        if new > 1:
            clean[row0:row0 + new] &= ~see[:, -1].to(DEV)[:, None, None]
        if new > 2:
            clean[row0:row0 + new, hq // 2:] &= ~see[:, -2].to(DEV)[:, None, None]
        row0 += new
    want, got = _compare(requests, cache, lines, q, out, hq, hkv, D, dtype, where=clean)
    assert not torch.isfinite(got[~clean].reshape(-1)).all() or clean.all()
    assert torch.equal(torch.isnan(want), torch.isnan(got))


def test_values_alone_not_finite():
    """Infinite values under finite scores: the infinity reaches the channel of the rows that see it and nothing else."""
    requests, D, page = [(37, 1, 2, 3), (0, 100, 0, 0)], 64, 32

    def poison(cache, lines, q):
        idx = U.offsets(D, page, "v").to(DEV)
        for line, s, value in ((lines[0], 40, math.inf), (lines[1], 50, -math.inf)):
            cache.value_pages[0].view(torch.bfloat16)[line[s // page], 0, idx[s % page][11]] = value

    cache, lines, q, out = _attend(requests, 2, 1, D, "bf16", page, poison=poison)
    rows = 107
    got = out[:rows, :2 * D].reshape(rows, 2, D)
    touched = torch.zeros((rows, 2, D), dtype=torch.bool, device=DEV)
    touched[3, :, 11] = True  # slot 40 is the last token of branch 0
    touched[7 + 50:, :, 11] = True
    assert torch.equal(torch.isinf(got), touched) and not torch.isnan(got).any()
    _compare(requests, cache, lines, q, out, 2, 1, D, "bf16", where=~touched)


@pytest.mark.parametrize("requests", [[(800, 1, 0, 0)], [(700, 100, 0, 0)]])
def test_extreme_scores(requests):
    """Queries a hundred times larger: one key takes nearly all of the weight, the reference of the exponents moves often; and keys of the type's
    lowest value, whose scores are minus infinity."""
    def poison(cache, lines, q):
        k = cache.key_pages[0].view(torch.bfloat16)
        k[lines[0][3]] = torch.finfo(torch.bfloat16).min
        q.copy_(q.abs() * 40)

    cache, lines, q, out = _attend(requests, 4, 4, 128, "bf16", 32, poison=poison)
    t = torch.bfloat16
    rows = U.new_rows(requests[0])
    want, mean_abs, _ = U.attention(requests, lines, cache.key_pages[0].view(t), cache.value_pages[0].view(t), q[:rows].reshape(rows, 4, 128), 4, 4, 128)
    got = out[:rows, :512].reshape(rows, 4, 128).double()
    # scores of up to 40 * 1.28^2 * 128 / sqrt(128) * 3 ~ 2300, fp32 sums of 128 products: 2^-24 * 128 * 6 * 2300 = 0.1 at the very worst
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 2 * (0.11 + 2.0 ** -8) * mean_abs).all()


def test_every_page_size_gives_the_same():
    requests, ref = [(333, 1, 2, 3), (10, 150, 0, 0)], None
    for page in (32, 64, 128, 256, 512, 1024):
        cache, lines, q, out = _attend(requests, 4, 2, 64, "bf16", page, seed=3)
        g = torch.Generator(device=DEV).manual_seed(17)
        for kind, pool in (("k", cache.key_pages), ("v", cache.value_pages)):
            idx = U.offsets(64, page, kind).to(DEV)
            for r, line in zip(requests, lines):
                total = r[0] + U.new_rows(r)
                x = torch.randn((total, 2, 64), generator=g, device=DEV).bfloat16()
                s = torch.arange(total, device=DEV)
                pid = torch.tensor(line, device=DEV)[s // page]
                for h in range(2):
                    pool[0].view(torch.bfloat16)[pid[:, None], h, idx[s % page]] = x[:, h]
        cache.attention(0, q, out[:, :256])
        ref = out.clone() if ref is None else ref
        assert torch.equal(ref, out)


def test_far_pages():
    """Pages whose elements lie beyond 2^32 bytes and 2^31 elements of the pool."""
    hq, hkv, D, page, dtype = 2, 2, 128, 1024, "bf16"
    n_pages = 9000  # 2 x 4.7 GB
    cache = B.PagedCache(U.shape_of(hq, hkv, D), n_pages=n_pages, max_requests=2, max_pages=3, max_rows=130, max_new=120, page_slots=page)
    lines = [[n_pages - 1, 3], [8500]]
    requests = [(1500, 1, 0, 0), (100, 120, 0, 0)]
    U.set_tables(cache, lines, [1, 2])
    cache.set_requests([1, 120], [0, 0], [0, 0], [1500, 100])
    for line in lines:
        for p in line:
            cache.key_pages[0, p].view(torch.bfloat16).normal_()
            cache.value_pages[0, p].view(torch.bfloat16).normal_()
    cache.plan()
    q, k, v = (torch.randn((130, 2, D), device=DEV).bfloat16() for _ in range(3))
    q0 = q.clone()
    cache.append(0, q, k, v)
    out = torch.full((130, hq * D), 9.0, dtype=torch.bfloat16, device=DEV)
    cache.attention(0, q, out)
    assert cache.status.item() == 0 and not torch.equal(q, q0)
    _compare(requests, cache, lines, q, out, hq, hkv, D, dtype)


def test_calls_that_do_nothing():
    """No plan, a plan of another batch, pages outside the pool."""
    requests = [(40, 1, 1, 2), (3, 80, 0, 0)]
    cache, lines = U.make(requests, 4, 2, 64, "bf16", 32)
    q = torch.randn((cache.max_rows, 4, 64), device=DEV).bfloat16()
    out = torch.full_like(q, 9.0)
    records = torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    cache.attention(0, q, out)
    assert cache.status.item() == B.PAGE_NO_PLAN and (out == 9.0).all()
    cache.status.zero_()
    cache.commit(records)
    assert cache.status.item() == B.PAGE_NO_PLAN and cache.cached.tolist() == [40, 3]
    cache.plan(1)
    cache._batch_c.n_requests = 2  # what the binding keeps a caller from doing
    cache.attention(0, q, out)
    assert cache.status.item() == B.PAGE_NO_PLAN and (out == 9.0).all()
    cache.plan()
    assert cache.status.item() == 0
    good = cache.attention(0, q, out).clone()
    cache.tables.block_table[0, 0] = cache.n_pages
    cache.tables.block_table[1, 1] = -5
    cache.attention(0, q, out)
    assert cache.status.item() == B.PAGE_BAD_PAGE
    assert torch.equal(out[83:], good[83:])


# --------------------------------------------------------------------------- commit
@pytest.mark.parametrize("hq,hkv,D,page,dtype", [(4, 2, 64, 32, "bf16"), (2, 2, 128, 64, "fp16"), (12, 3, 128, 32, "bf16")])
def test_commit(hq, hkv, D, page, dtype):
    requests = [(30, 1, 3, 5), (0, 50, 0, 0), (63, 1, 2, 9), (12, 0, 4, 3), (5, 2, 1, 7), (31, 1, 2, 2), (0, 0, 0, 0), (40, 1, 3, 3), (40, 1, 3, 3), (8, 1, 2, 4), (90, 1, 2, 40)]
    records = [(2, 4, 9, 0), (1, 7, 9, 0), (1, 9, 9, 0), (3, 1, 9, 0), (0, 6, 9, 0), (-1, 0, 9, 0), (0, 0, 0, 0), (-1, 0, -1, 0), (3, 1, 9, 0), (1, 5, 9, 0), (1, 40, 9, 0)]
    bad = {8, 9}  # no such branch, more tokens than it has
    cache, lines = U.make(requests, hq, hkv, D, dtype, page, layers=3)
    cache.plan()
    keys, values = cache.key_pages.clone(), cache.value_pages.clone()
    rec = torch.tensor(records, dtype=torch.int32, device=DEV)
    cached = torch.full((len(requests) + 2,), -3, dtype=torch.int32, device=DEV)
    cache.commit(rec, cached)
    assert cache.status.item() == B.PAGE_BAD_RECORD
    after, ik, iv = [], U.offsets(D, page, "k").to(DEV), U.offsets(D, page, "v").to(DEV)
    for r, ((c, trunk, n, k), (b, a, token, _)) in enumerate(zip(requests, records)):
        if n * k == 0:
            after.append(c + trunk)
            continue
        if r in bad or (b < 0 and token < 0):
            after.append(c)
            continue
        after.append(c + trunk + (a if b >= 0 else 0))
        for j in range(a if b > 0 else 0):
            s, d = c + trunk + b * k + j, c + trunk + j
            for pool, idx in ((keys, ik), (values, iv)):
                pool[:, lines[r][d // page], :, idx[d % page]] = pool[:, lines[r][s // page], :, idx[s % page]]
    assert cached.tolist() == after + [-3, -3]
    assert torch.equal(keys, cache.key_pages) and torch.equal(values, cache.value_pages)
    assert cache.cached[:len(requests)].tolist() == [r[0] for r in requests]
    cache.commit(rec)  # again, in place
    assert cache.cached.tolist() == after
    assert torch.equal(keys, cache.key_pages) and torch.equal(values, cache.value_pages)


# --------------------------------------------------------------------------- steps
class Model:
    """One attention layer's worth of a step in 64 bits: per request the rows of its keys and values, as the cache holds them."""

    def __init__(self, n):
        self.k, self.v = [None] * n, [None] * n


def _step_lengths(step):
    return [[(0, 37, 0, 0), (0, 120, 0, 0), (0, 5, 0, 0)],
            [(None, 1, 2, 4), (None, 1, 3, 3), (None, 30, 0, 0)],
            [(None, 1, 1, 6), (None, 1, 0, 0), (None, 1, 2, 5)],
            [(None, 1, 2, 4), (None, 0, 0, 0), (None, 1, 1, 1)]][step]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_steps_together(dtype):
    """Four steps of three requests: plan, append, attention, sampling of one request's branches, commit.  After every step the cache's rows are what
    the commits say, and the attention is that of the formula over them."""
    hq, hkv, D, page, theta, V = 8, 2, 64, 32, 10000.0, 300
    t = U.TYPES[dtype]
    cache = B.PagedCache(U.shape_of(hq, hkv, D, 1, theta), n_pages=20, max_requests=3, max_pages=10, max_rows=200, max_new=150, page_slots=page, dtype=dtype)
    g = torch.Generator(device=DEV).manual_seed(5)
    held_k, held_v = [torch.empty((0, hkv, D), dtype=t, device=DEV) for _ in range(3)], [torch.empty((0, hkv, D), dtype=t, device=DEV) for _ in range(3)]
    for step in range(4):
        requests = [(len(held_k[r]), *spec[1:]) for r, spec in enumerate(_step_lengths(step))]
        cache.set_requests([r[1] for r in requests], [r[2] for r in requests], [r[3] for r in requests])
        cache.plan()
        assert cache.status.item() == 0 and cache.cached.tolist() == [r[0] for r in requests]
        rows = sum(map(U.new_rows, requests))
        assert cache.row_start[3].item() == rows
        q, k, v = ((torch.randn((200, h, D), generator=g, device=DEV) * 1.28).to(t) for h in (hq, hkv, hkv))
        cache.append(0, q, k, v)
        out = torch.full((200, hq * D), 9.0, dtype=t, device=DEV)
        cache.attention(0, q, out)
        lines = [line[:h] for line, h in zip(cache.tables.block_table.tolist(), cache.tables.held.tolist())]
        assert len({p for line in lines for p in line}) == sum(map(len, lines)) == 20 - cache.tables.free_count.item()
        # what the cache holds is what was committed, and the new rows behind it
        records = []
        for r, request in enumerate(requests):
            total = request[0] + U.new_rows(request)
            K, Vv = (U.rows_of(p[0].view(t), lines[r], D, kind)[:, :total].transpose(0, 1) for p, kind in ((cache.key_pages, "k"), (cache.value_pages, "v")))
            assert torch.equal(K[:request[0]], held_k[r]) and torch.equal(Vv[:request[0]], held_v[r])
            row0 = cache.row_start[r].item()
            assert torch.equal(Vv[request[0]:], v[row0:row0 + U.new_rows(request)])
            n, kk = request[2], request[3]
            if n * kk:
                logits = torch.randn((request[1] + n * kk, V), generator=g, device=DEV)
                draft = torch.softmax(torch.randn((n, kk, V), generator=g, device=DEV), -1)
                got = B.spec_sample(logits, torch.randn(V, generator=g, device=DEV), torch.randint(0, V, (n, kk), generator=g, device=DEV).int(), draft,
                                    torch.rand((n, kk + 1), generator=g, device=DEV) * 0.05, has_root=request[1] > 0, prefix_len=request[0])
                record = [got["selected"], got["commit_len"], got["commit_token"], got["new_prefix_len"]]
            else:
                record = [-1, 0, 7, 0]
            records.append(record)
            keep = list(range(request[0] + request[1])) + [request[0] + request[1] + max(record[0], 0) * kk + j for j in range(record[1])]
            held_k[r], held_v[r] = K[keep].clone(), Vv[keep].clone()
        _compare(requests, cache, lines, q, out, hq, hkv, D, dtype)
        cache.commit(torch.tensor(records, dtype=torch.int32, device=DEV))
        assert cache.cached.tolist() == [len(x) for x in held_k]
    # requests that end give their pages back
    cache.cached.zero_()
    cache.set_requests([0, 0, 0], [0, 0, 0], [0, 0, 0])
    cache.plan()
    assert cache.tables.free_count.item() == 20 and sorted(cache.tables.free_pages.tolist()) == list(range(20))


def test_a_captured_step_serves_other_lengths():
    """Plan, append, attention and commit of a step in a graph, replayed on other lengths and rows, against the same calls made eagerly."""
    hq, hkv, D, page = 8, 2, 128, 32

    def fresh():
        c = B.PagedCache(U.shape_of(hq, hkv, D), n_pages=300, max_requests=4, max_pages=100, max_rows=160, max_new=120, page_slots=page)
        return c, [torch.zeros((160, h, D), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv, hq, hq)], torch.zeros((4, 4), dtype=torch.int32, device=DEV)

    def calls(c, m, records):
        c.plan()
        c.append(0, m[0], m[1], m[2], m[3])
        c.attention(0, m[3], m[4])
        c.commit(records)

    (cg, mg, rg), (ce, me, re) = fresh(), fresh()
    calls(cg, mg, rg)  # requests that bring nothing
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(cg, mg, rg)
    g = torch.Generator(device=DEV).manual_seed(2)
    for trunk, n, k, record in [([100, 1, 7, 0], [0, 0, 0, 0], [0, 0, 0, 0], [[-1, 0, 1, 0]] * 4),
                                ([1, 110, 1, 3], [2, 0, 3, 0], [3, 0, 2, 0], [[1, 2, 5, 0], [-1, 0, 4, 0], [2, 2, 1, 0], [-1, 0, 1, 0]]),
                                ([1, 1, 1, 1], [0, 2, 0, 1], [0, 9, 0, 4], [[-1, 0, 1, 0], [1, 9, 1, 0], [-1, 0, 1, 0], [0, 4, 1, 0]]),
                                ([0, 1, 120, 0], [0, 0, 0, 0], [0, 0, 0, 0], [[-1, 0, 1, 0]] * 4)]:
        for c, m, r in ((cg, mg, rg), (ce, me, re)):
            c.set_requests(trunk, n, k)
            r.copy_(torch.tensor(record, dtype=torch.int32))
        for a, b in zip(mg[:3], me[:3]):
            a.copy_(torch.randn(a.shape, generator=g, device=DEV).bfloat16())
            b.copy_(a)
        graph.replay()
        calls(ce, me, re)
        torch.cuda.synchronize()
        assert cg.status.item() == ce.status.item() == 0
        for a, b in zip((*mg, *cg.tables.tensors(), cg.cached, cg.slot, cg.key_pages, cg.value_pages), (*me, *ce.tables.tensors(), ce.cached, ce.slot, ce.key_pages, ce.value_pages)):
            assert torch.equal(a, b)


def test_other_streams_and_repeats():
    requests = STEPS["mixed"]
    cache, lines, q, out = _attend(requests, 8, 2, 128, "bf16", 64)
    again = torch.full_like(out, 9.0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        cache.plan()
        cache.attention(0, q, again[:, :1024])
    stream.synchronize()
    assert torch.equal(out, again)


def test_two_caches_on_two_streams():
    """Steps of two caches enqueued in turn on streams of their own give what each gives alone."""
    steps = [_attend(STEPS[name], 8, 2, 128, "bf16", 64, seed=i) for i, name in enumerate(("mixed", "long_chunk"))]
    streams, again = [torch.cuda.Stream() for _ in steps], [torch.full_like(s[3], 9.0) for s in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        for (cache, _, q, _), stream, out in zip(steps, streams, again):
            with torch.cuda.stream(stream):
                cache.plan()
                cache.attention(0, q, out[:, :1024])
    torch.cuda.synchronize()
    for (cache, _, _, out), other in zip(steps, again):
        assert cache.status.item() == 0 and torch.equal(out, other)
