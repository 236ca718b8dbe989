"""Key ranges so long that the attention kernels fetch page ids more than once, and plans whose requests are spread over several workgroups.

The attention's cases need no large pools: a few pages without weight fill long block tables, and every probed block is a page of its own.  Page
p < PROBES has a key in channel p and values of one in channel p; a query with one channel alone looks for the page of that channel, and its output is
one there and zero elsewhere, unless keys or values of that block were read from another place."""
import random

import pytest

torch = pytest.importorskip("torch")

import paged_util as U
from paper_2503_00784_amd import binding as B
from test_gpu_paged import _check_plan, _planner, say
from test_paged import _cut

DEV = "cuda:0"
PROBES, FILL = 48, 4
# name -> requests (cached, trunk, n, k), kv heads, query heads, least blocks of a streamed request's range, of a tiled one's
CASES = {
    "rows_in_registers": ([(70000, 1, 0, 0)] * 4, 64, 64, 4 * 129, 0),           # each of four waves goes through 64 ids more than twice
    "rows_in_registers_grouped": ([(150000, 2, 0, 0)] * 8, 8, 32, 4 * 65, 0),
    "teams_of_one_wave": ([(17700, 20, 0, 0)] * 4, 64, 64, 2 * 129, 0),          # one team or two
    "teams_of_two_waves": ([(17650, 2, 2, 30)] * 4, 64, 64, 2 * 129, 0),
    "tiles": ([(7200, 1030, 0, 0)], 32, 32, 0, 257),                             # two blocks a stage
    "prompt": ([(0, 8272, 0, 0)], 8, 8, 0, 257),                                 # the last tile has a wave without rows
    "all_kinds": ([(25600, 1, 0, 0), (25590, 1, 1, 30), (25580, 1, 2, 20), (100, 150, 0, 0)], 64, 64, 4 * 65, 0),
}


def _ranges(requests, hkv, hq):
    """(blocks of a streamed request's range, of a tiled one's) by the rules that the plan goes by, 0 without one; requests of a kind are cut alike."""
    group = hq // hkv
    rows = [(r[0], U.new_rows(r)) for r in requests]
    cut = _cut(rows, max(n for _, n in rows), (max(c + n for c, n in rows) + 31) // 32 + 1, hq, hkv)
    out = []
    for kind in ("stream_items", "tile_items"):
        mine = [(c, n) for c, n in rows if (n * group <= 64) == (kind == "stream_items")]
        tiles = sum(1 if kind == "stream_items" else -(-n * group // 128) for _, n in mine)
        chunks = cut[kind] // max(1, tiles)
        assert chunks * tiles == cut[kind]
        out.append(min(-(-((c + n + 31) // 32) // chunks) for c, n in mine) if mine else 0)
    return out


@pytest.mark.parametrize("name", list(CASES))
def test_the_ranges_are_long(name):
    requests, hkv, hq, streamed, tiled = CASES[name]
    got = _ranges(requests, hkv, hq)
    assert got[0] >= streamed and got[1] >= tiled, got


def _probed(request, r, length, group, D):
    """The blocks to look at: the first and last of every range and those where a wave, a team or a stage comes to its next 64 ids."""
    rows, blocks = U.new_rows(request), (request[0] + U.new_rows(request) + 31) // 32
    rng = random.Random(r)
    step = 4 if rows * group <= 16 else 2 if rows * group > 64 or D == 64 else 1
    edges = {b for c in range(0, blocks, length or blocks) for i in (0, 63, 64, 65, 127, 128, 129) for b in range(c + i * step - 1, c + i * step + step + 1)}
    edges = sorted(b for b in edges | {blocks - 1} if 0 <= b < blocks)
    rest = [b for b in range(blocks) if b not in set(edges)]
    chosen = rng.sample(edges, min(PROBES, len(edges)))
    return chosen + rng.sample(rest, min(PROBES - len(chosen), len(rest)))


@pytest.mark.gpu
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("name", list(CASES))
def test_attention_of_long_ranges(name, D, dtype):
    requests, hkv, hq, _, _ = CASES[name]
    say(name, D, dtype)
    t, page, n_pages = U.TYPES[dtype], 32, PROBES + FILL
    rows = sum(map(U.new_rows, requests))
    need = [-(-(r[0] + U.new_rows(r)) // page) for r in requests]
    cache = B.PagedCache(U.shape_of(hq, hkv, D), n_pages=n_pages, max_requests=len(requests), max_pages=max(need), max_rows=rows + 3,
                         max_new=max(map(U.new_rows, requests)), page_slots=page, dtype=dtype)
    lengths = _ranges(requests, hkv, hq)
    g = torch.Generator().manual_seed(len(name))
    table = torch.randint(PROBES, n_pages, (len(requests), max(need)), generator=g, dtype=torch.int32)
    probes = []
    for r, request in enumerate(requests):
        probes.append(_probed(request, r, lengths[0 if U.new_rows(request) * (hq // hkv) <= 64 else 1], hq // hkv, D))
        for p, b in enumerate(probes[-1]):
            table[r, b] = p
    cache.tables.block_table.copy_(table)
    cache.tables.held.copy_(torch.tensor(need, dtype=torch.int32))
    cache.tables.free_count.zero_()
    ik, iv = U.offsets(D, page, "k"), U.offsets(D, page, "v")
    keys, values = torch.zeros((n_pages, hkv, page * D)), torch.zeros((n_pages, hkv, page * D))
    for p in range(PROBES):
        keys[p][:, ik[:, p]] = 30.0
        values[p][:, iv[:, p]] = 1.0
    cache.key_pages[0].view(t).copy_(keys)
    cache.value_pages[0].view(t).copy_(values)
    # row i, head h looks for the page of channel (i + h) mod PROBES: its keys score 30, all others 0
    look = (torch.arange(cache.max_rows)[:, None] + torch.arange(hq)[None]) % PROBES
    q = torch.nn.functional.one_hot(look, D).to(t).to(DEV) * 8.0
    cache.set_requests([r[1] for r in requests], [r[2] for r in requests], [r[3] for r in requests], [r[0] for r in requests])
    cache.plan()
    assert cache.status.item() == 0
    out = torch.full((cache.max_rows, hq, D), 9.0, dtype=t, device=DEV)
    cache.attention(0, q, out, 0.125)
    assert cache.status.item() == 0 and (out[rows:] == 9.0).all()
    got, row0, checked = out.cpu().double(), 0, 0
    for r, request in enumerate(requests):
        new = U.new_rows(request)
        see = U.visible(request)
        block_seen = torch.zeros((new, PROBES), dtype=torch.bool)
        for p, b in enumerate(probes[r]):
            block_seen[:, p] = see[:, 32 * b:32 * b + 32].any(-1)
        mine, at = got[row0:row0 + new], look[row0:row0 + new]
        sees = block_seen.gather(1, at)  # [new][hq]: the row sees some key of the page that it looks for
        want = torch.nn.functional.one_hot(at, D).double()
        # What is found has at least one key of weight 1; up to 150002 others have e^-30 = 1e-13 each, 1.4e-8 in all.  Weights and output are rounded once
        # each, u, the quotient in fp32.
        err = (mine - want).abs()[sees]
        assert err.numel() and float(err.max()) <= 2.1 * torch.finfo(t).eps / 2 + 2.0 ** -20, (r, [probes[r][p] for p in at[sees][err.amax(-1) > 0.01][:9].tolist()])
        checked += int(sees.sum())
        row0 += new
    say("rows and heads that found their page:", checked)


# --------------------------------------------------------------------------- plans
def _spread_inputs(R, longest, page, seed):
    """Requests of up to `longest` new rows that hold the pages of what they have cached and some more, or are to be given many; some release all they hold."""
    rng = random.Random(seed)
    requests, held = [], []
    for r in range(R):
        kind = rng.randrange(4)
        if kind == 0:
            requests.append((0, 0, 0, 0))
            held.append(rng.randint(0, 2 * longest // page))
            continue
        cached = rng.choice([0, rng.randint(0, 3000)])
        requests.append((cached, rng.randint(1, longest), 0, 0) if kind == 1 else (cached, 1, rng.randint(0, 3), rng.randint(0, 9)))
        held.append(-(-cached // page) + rng.choice([0, 0, 1, rng.randint(0, 60)]))
    requests[R // 2] = (77, longest, 0, 0)
    held[R // 2] = 77 // page + 1
    need = [-(-(q[0] + U.new_rows(q)) // page) for q in requests]
    n_pages = max(sum(need), sum(held)) + rng.randint(0, 5)
    ids = list(range(n_pages))
    rng.shuffle(ids)
    lines, at = [], 0
    for h in held:
        lines.append(ids[at:at + h])
        at += h
    return requests, lines, ids[at:], n_pages, max(max(need), max(held))


# room for more columns than 512 or 8192, or new rows beyond: up to 16 workgroups a request
@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("R,longest,page,columns", [(9, 513, 32, 0), (20, 1500, 32, 0), (40, 300, 32, 700), (30, 5000, 64, 0), (12, 9000, 32, 0), (150, 8193, 128, 0),
                                                    (1500, 1100, 32, 0), (9, 40, 32, 8193)])
def test_plan_of_spread_requests(R, longest, page, columns, in_place):
    requests, lines, free, n_pages, max_pages = _spread_inputs(R, longest, page, R)
    want = U.plan(requests, page, (lines, free), sum(map(U.new_rows, requests)) + 4)
    cache = _planner(requests, lines, free, n_pages, max(max_pages, columns), page)
    assert max(cache.max_new, cache.max_pages) > 512 and R > 8
    say(R, longest, "pages released", sum(max(0, len(l) - len(w)) for l, w in zip(lines, want[3])), "taken", sum(max(0, len(w) - len(l)) for l, w in zip(lines, want[3])))
    if in_place:
        cache.plan()
    else:
        source = B.PageTables(*[x.clone() for x in cache.tables.tensors()])
        before = [x.clone() for x in source.tensors()]
        for x in cache.tables.tensors():
            x.fill_(-7)
        cache.plan(source=source)
        for a, b in zip(before, source.tensors()):
            assert torch.equal(a, b)
    _check_plan(cache, want, cache.tables)
