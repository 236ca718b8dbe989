"""Plain 64-bit implementations of the paged-cache calls and helpers shared by their tests (not collected by pytest)."""
import math

import torch

from paper_2503_00784_amd import binding as B
from paper_2503_00784_amd import inputs

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def shape_of(hq, hkv, D, layers=1, theta=10000.0):
    return inputs.ModelShape(layers, 64 * hq, hq, hkv, D, 64, 1000, rope_theta=theta)


def new_rows(r):
    return r[1] + r[2] * r[3]


def plan(requests, page, tables, max_rows):
    """(row_start, position, slot, block table lines, held, free stack) of requests [(cached, trunk, n, k)]; tables: (lines, free), each
    line holding the request's pages."""
    lines, free = tables
    need = [-(-(r[0] + new_rows(r)) // page) for r in requests]
    stack = list(free)
    for line, m in zip(lines, need):
        stack += line[m:]
    out, row_start, position, slot = [], [0], [], []
    for (cached, trunk, n, k), line, m in zip(requests, lines, need):
        line = list(line[:m])
        while len(line) < m:
            line.append(stack.pop())
        for t in range(trunk + n * k):
            position.append(cached + t if t < trunk else cached + trunk + (t - trunk) % k)
            slot.append(line[(cached + t) // page] * page + (cached + t) % page)
        row_start.append(len(slot))
        out.append(line)
    pad = [-1] * (max_rows - len(slot))
    return row_start, position + pad, slot + pad, out, need, stack


def visible(request):
    """[new rows][slots]: what every row sees."""
    cached, trunk, n, k = request
    new = trunk + n * k
    see = torch.zeros((new, cached + new), dtype=torch.bool)
    see[:, :cached] = True
    for t in range(new):
        if t < trunk:
            see[t, cached:cached + t + 1] = True
        else:
            i, j = divmod(t - trunk, k)
            see[t, cached:cached + trunk] = True
            see[t, cached + trunk + i * k:cached + trunk + i * k + j + 1] = True
    return see


def make(requests, hq, hkv, D, dtype="bf16", page=32, layers=1, device="cuda:0", seed=0, theta=10000.0, spare=3, pad=3, max_new=None):
    """A PagedCache with the pages of `requests` dealt at random, its tables filled in for the planned step (not planned yet), and its keys and
    values drawn at random, stale slots included."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-(r[0] + new_rows(r)) // page) for r in requests]
    n_pages = sum(need) + spare
    rows = sum(map(new_rows, requests))
    cache = B.PagedCache(shape_of(hq, hkv, D, layers, theta), n_pages=n_pages, max_requests=len(requests), max_pages=max(need) + 1, max_rows=rows + pad,
                         max_new=max(1, max(map(new_rows, requests))) if max_new is None else max_new, page_slots=page, dtype=dtype, device=device)
    order = torch.randperm(n_pages, generator=g).tolist()
    lines, at = [], 0
    for m in need:
        lines.append(order[at:at + m])
        at += m
    set_tables(cache, lines, order[at:])
    cache.set_requests([r[1] for r in requests], [r[2] for r in requests], [r[3] for r in requests], [r[0] for r in requests])
    for pool in (cache.key_pages, cache.value_pages):
        pool.view(TYPES[dtype]).copy_(torch.randn(pool.shape, generator=g) * 1.28)
    return cache, lines


def set_tables(cache, lines, free):
    t = cache.tables
    table = torch.full(tuple(t.block_table.shape), -1, dtype=torch.int32)
    for r, line in enumerate(lines):
        table[r, :len(line)] = torch.tensor(line, dtype=torch.int32)
    t.block_table.copy_(table)
    held = torch.zeros(cache.max_requests, dtype=torch.int32)
    held[:len(lines)] = torch.tensor([len(x) for x in lines], dtype=torch.int32)
    t.held.copy_(held)
    stack = torch.full((cache.n_pages,), -1, dtype=torch.int32)
    stack[:len(free)] = torch.tensor(free, dtype=torch.int32)
    t.free_pages.copy_(stack)
    t.free_count.fill_(len(free))


def offsets(D, page, kind):
    """[page][D]: place of (slot, channel) in a page plane, from the library's own map of the cache."""
    f = B.load().duo_k_cache_offset if kind == "k" else B.load().duo_v_cache_offset
    return torch.tensor([[f(D, s, d) for d in range(D)] for s in range(page)])


def rows_of(pool, lines_r, D, kind):
    """Keys or values of one request as [kv heads][slots][D]; pool [pages][kv heads][page * D] of one layer."""
    page = pool.shape[-1] // D
    x = pool[torch.tensor(lines_r, device=pool.device)]
    idx = offsets(D, page, kind).reshape(-1).to(pool.device)
    return x[..., idx].reshape(len(lines_r), pool.shape[1], page, D).transpose(0, 1).reshape(pool.shape[1], -1, D)


def attention(requests, lines, keys, values, q, hq, hkv, D, scale=None):
    """(out, mean |v| under the weights, largest scale * sum |q k| of a row), [rows][hq][D] and [rows][hq] in 64 bits on the tensors' device."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, weight, size, row0 = [], [], [], 0
    for r, request in enumerate(requests):
        new = new_rows(request)
        if new == 0:
            continue
        total = request[0] + new
        K, V = (rows_of(p, lines[r], D, kind)[:, :total].double() for p, kind in ((keys, "k"), (values, "v")))
        see = visible(request).to(q.device)
        x = q[row0:row0 + new].double()
        o, a, s_max = torch.empty_like(x), torch.empty_like(x), torch.empty((new, hq), dtype=torch.float64, device=q.device)
        for h in range(hq):
            kv = h // (hq // hkv)
            s = ((x[:, h] @ K[kv].T.contiguous()) * scale).masked_fill(~see, -math.inf)
            p = torch.softmax(s, -1)
            # what a row does not see does not touch it, infinities and NaN included
            if torch.isfinite(V[kv]).all():
                o[:, h], a[:, h] = p @ V[kv], p @ V[kv].abs()
            else:
                for t in range(new):
                    o[t, h], a[t, h] = p[t, see[t]] @ V[kv][see[t]], p[t, see[t]] @ V[kv][see[t]].abs()
            size = (x[:, h].abs() @ K[kv].abs().T.contiguous()) * scale
            s_max[:, h] = size.masked_fill(~see, 0.0).amax(-1)
        out.append(o)
        weight.append(torch.stack([a, s_max[..., None].expand_as(a)]))
        row0 += new
    w = torch.cat(weight, 1)
    return torch.cat(out), w[0], w[1]


def attention_bound(out, mean_abs, size, dtype, D, keys, v_max, pairs):
    """How far the kernel may be off.  With u half a step of the 16-bit type:
      - the output is rounded once: u |o|;
      - a softmax weight is rounded once (u) or kept as a pair (u^2); in fp16 weights below the normal range are off by up to 2^-25 each, next to a sum
        of at least 1 (the reference of the exponents is the score of a key);
      - scores are fp32 sums of D products: D 2^-24 sum |q k| each, the exponent and its argument 2^-23 of up to 2 size + 8;
      - sums over the keys are fp32: keys 2^-24.
    A relative error e of every weight moves o by at most 2 e times the weighted mean of |v|."""
    u = torch.finfo(TYPES[dtype]).eps / 2
    e = (u * u if pairs else u) + 1.5 * (D * 2.0 ** -24 * size + 2.0 ** -23 * (2 * size + 16)) + keys * 2.0 ** -23
    tiny = keys * 2.0 ** -24 * v_max if dtype == "fp16" else 0.0
    return u * out.abs() * (1 + u) + (1 + u) * (2 * e * mean_abs + tiny) + 1e-30
