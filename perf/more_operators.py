"""Products on weights held in 8-bit floating point and mixture-of-experts layers, as cases to be timed and compared.

product: y = x W^T with W held as e4m3 with one power-of-two scale for every block of 128 x 128, x given in 16 bits and brought to
e4m3 on the way with a scale for every 128 values of a row.  The scale of a block is the smallest power of two that brings its
largest magnitude to 448, e4m3's largest value, or below.

experts: a whole layer of experts for the few rows of a verify step.  The router's logits x R^T choose the top_k experts of a row
(equal ones by ascending index), their softmax weights (over all experts, or over the chosen ones where `renormalise` is set) the
shares of silu(x G^T) * (x U^T) D^T in the row's output.  The experts' matrices are held in 16 bits or (`scaled`) in the blocks
above; the rows are not brought to 8 bits here.  Rows of a padded step whose position is -1 are left as they are.

`run` makes the calls of the framework where `own` is true and computes the same from elementary torch operations otherwise;
`exact` is the same again in 64 bits.  Sizes follow from the case alone, values from the seed.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
BLOCK = 128
LARGEST = 448.0   # of e4m3


def _product(name, rows, n, k, dtype, fp32=False):
    return {"name": name, "op": "product", "rows": rows, "n": n, "k": k, "dtype": dtype, "fp32": fp32}


def _experts(name, rows, experts, top_k, d, ff, dtype, scaled, renormalise=True, idle=0):
    return {"name": name, "op": "experts", "rows": rows, "experts": experts, "top_k": top_k, "d": d, "ff": ff, "dtype": dtype, "scaled": scaled,
            "renormalise": renormalise, "idle": idle}


def listed():
    return [
        # the output projection of the 7B shape for one token: the smallest stream, latency counts
        _product("product_single", 1, 4096, 4096, "bf16"),
        # the down projection of the 7B shape for a root token and eight draft tokens, the paper's own precision
        _product("product_step", 9, 4096, 11008, "fp16"),
        # gate and up of the 7B shape for a root token and four branches of eight
        _product("product_verify", 33, 22016, 4096, "bf16"),
        # the LM head of the 8B shape, its logits in 32 bits as the sampler takes them
        _product("product_head", 17, 128256, 4096, "bf16", fp32=True),
        # a prompt chunk through the down projection of the 13B shape, an odd number of rows
        _product("product_chunk", 999, 5120, 13824, "fp16"),
        # packed prompts through gate and up of the 8B shape: the matrix units
        _product("product_prompts", 4111, 28672, 4096, "bf16"),
        # a few small experts, one for each row: launches are what counts
        _experts("experts_small", 3, 4, 1, 768, 1408, "fp16", scaled=True),
        # a single token on many small experts held in 16 bits
        _experts("experts_single", 1, 64, 6, 2048, 1408, "bf16", scaled=False),
        # a root token and eight draft tokens on a few large experts held in 8 bits
        _experts("experts_step", 9, 8, 2, 4096, 14336, "bf16", scaled=True),
        # four branches of eight behind their root token in a step padded to 37 rows, shares as the softmax over all experts has them
        _experts("experts_verify", 37, 32, 4, 2048, 2816, "fp16", scaled=False, renormalise=False, idle=4),
        # as many rows as a verify step takes, on a hundred experts and more: nearly every one is chosen
        _experts("experts_many", 80, 128, 8, 4096, 1536, "bf16", scaled=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [work(c) for c in listed()]
    limit = {key: max(w[key] for w in most) for key in ("bytes", "flops")}
    while True:
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        if rng.random() < 0.5:
            rows = rng.choice([_log_int(rng, 1, 80), _log_int(rng, 1, 80), _log_int(rng, 81, 5000)])
            case = _product("", rows, _log_int(rng, 40, 60000), 32 * _log_int(rng, 2, 500), dtype, rng.random() < 0.25)
        else:
            experts = _log_int(rng, 2, 256)
            rows = _log_int(rng, 1, 80)
            case = _experts("", rows, experts, rng.randint(1, min(experts, 8)), 64 * _log_int(rng, 4, 110), 32 * _log_int(rng, 4, 450), dtype,
                            rng.random() < 0.5, rng.random() < 0.7, rng.choice([0, 0, rng.randint(0, rows - 1)]))
            if 3.0 * experts * case["d"] * case["ff"] > 2.5e9:
                continue
        w = work(case)
        if w["bytes"] <= limit["bytes"] and w["flops"] <= limit["flops"]:
            del case["name"]
            return case


# --------------------------------------------------------------------------- inputs
def _gen(seed, *stream):
    g = torch.Generator(device=DEVICE)
    key = int(seed) & 0x7FFFFFFF
    for s in stream:
        key = (key * 1000003 + int(s) + 12345) & 0x7FFFFFFFFFFF
    g.manual_seed(key)
    return g


def _type(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _rows(case, width, seed):
    """Normalised rows with a few channels that stand out, as they do behind a norm's gains."""
    g = _gen(seed, 1)
    gain = 1.0 + 0.1 * torch.randn(width, generator=g, device=DEVICE)
    gain = torch.where(torch.rand(width, generator=g, device=DEVICE) < 0.003, 12.0 * gain, gain)
    return (torch.randn((case["rows"], width), generator=g, device=DEVICE) * gain).to(_type(case))


def _weights(case, n, k, seed, *stream):
    """[n][k] with outputs of the inputs' size; rows differ in their norms."""
    g = _gen(seed, 2, *stream)
    norm = torch.exp(0.3 * torch.randn((n, 1), generator=g, device=DEVICE)) / math.sqrt(k)
    return (torch.randn((n, k), generator=g, device=DEVICE) * norm).to(_type(case))


def _router(case, seed):
    return _weights(case, case["experts"], case["d"], seed, 9)


def _expert(case, e, seed):
    """Gate, up and down matrices of one expert."""
    d, ff = case["d"], case["ff"]
    return _weights(case, ff, d, seed, 3, e), _weights(case, ff, d, seed, 4, e), _weights(case, d, ff, seed, 5, e)


def _positions(case, seed):
    """Rotary positions of a padded step's rows, -1 behind its last row; None where every row counts."""
    if not case["idle"]:
        return None
    live = case["rows"] - case["idle"]
    return torch.tensor([100 + t for t in range(live)] + [-1] * case["idle"], dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    state = {"case": case}
    if case["op"] == "product":
        state["x"] = _rows(case, case["k"], seed)
        w = _weights(case, case["n"], case["k"], seed)
        if own:
            from paper_2503_00784_amd import binding as B
            state["matrix"] = B.ScaledMatrix(w)
        else:
            state["matrix"] = _plain_blocks(w, BLOCK)
        state["out"] = torch.zeros((case["rows"], (case["n"] + 7) // 8 * 8), dtype=torch.float32 if case["fp32"] else _type(case), device=DEVICE)[:, :case["n"]]
        return state
    state["x"] = _rows(case, case["d"], seed)
    state["position"] = _positions(case, seed)
    state["out"] = torch.zeros_like(state["x"])
    router = _router(case, seed)
    experts = (_expert(case, e, seed) for e in range(case["experts"]))
    if own:
        from paper_2503_00784_amd import binding as B
        state["layer"] = B.ExpertLayer(router, experts, case["top_k"], scaled=case["scaled"], renormalise=case["renormalise"])
    else:
        state["router"] = router
        state["weights"] = [tuple(_plain_blocks(w, BLOCK) if case["scaled"] else w for w in e) for e in experts]
    return state


# --------------------------------------------------------------------------- one pass
def run(state):
    if state["case"]["op"] == "product":
        if own:
            return state["matrix"].product(state["x"], state["out"])
        return _plain_product(state)
    if own:
        y, experts, gates = state["layer"].run(state["x"], state["out"], position=state["position"])
        if state["position"] is not None:
            live = state["case"]["rows"] - state["case"]["idle"]
            experts, gates = experts[:live], gates[:live]
        return {"y": y, "experts": experts, "gates": gates}
    return _plain_experts(state)


def _plain_blocks(x, rows):
    """x [n][k] in blocks of `rows` x 128: (e4m3 values, a power of two for every block), both as they are kept."""
    n, k = x.shape
    pad_n, pad_k = -n % rows, -k % BLOCK
    v = torch.nn.functional.pad(x.float(), (0, pad_k, 0, pad_n)).reshape((n + pad_n) // rows, rows, (k + pad_k) // BLOCK, BLOCK)
    mantissa, exponent = torch.frexp(v.abs().amax((1, 3)))       # mantissa in [1/2, 1); 448 = 7/8 * 2^9
    exponent = torch.where(mantissa == 0, 0, exponent - 9 + (mantissa > 0.875).int())
    scale = torch.ldexp(torch.ones_like(mantissa), exponent)
    q = (v / scale[:, None, :, None]).reshape(n + pad_n, k + pad_k)[:n, :k].to(torch.float8_e4m3fn)
    return q, scale


def _plain_values(blocks, rows):
    q, scale = blocks
    n, k = q.shape
    return q.float() * scale.repeat_interleave(rows, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]


def _plain_product(state):
    x = _plain_values(_plain_blocks(state["x"], 1), 1)
    w = _plain_values(state["matrix"], BLOCK)
    state["out"].copy_(torch.matmul(x, w.t()))
    return state["out"]


def _plain_experts(state):
    case, out = state["case"], state["out"]
    live = case["rows"] - case["idle"]
    x = state["x"][:live]
    # 64 bits: which of two experts with nearly equal logits a row takes decides its whole output
    logits = torch.matmul(x.double(), state["router"].double().t())
    order = torch.sort(logits, dim=-1, descending=True, stable=True)
    chosen, value = order.indices[:, :case["top_k"]], order.values[:, :case["top_k"]]
    share = torch.exp(value - order.values[:, :1])
    share = share / (share if case["renormalise"] else torch.exp(logits - order.values[:, :1])).sum(-1, keepdim=True)
    share = share.float()
    y = torch.zeros((live, case["d"]), dtype=torch.float32, device=DEVICE)
    xf = x.float()
    for e, matrices in enumerate(state["weights"]):
        row, slot = torch.nonzero(chosen == e, as_tuple=True)
        if len(row) == 0:
            continue
        gate, up, down = (_plain_values(m, BLOCK) if case["scaled"] else m.float() for m in matrices)
        a, b = torch.matmul(xf[row], gate.t()), torch.matmul(xf[row], up.t())
        h = a / (1.0 + torch.exp(-a)) * b * share[row, slot, None]
        y[row] += torch.matmul(h, down.t())
    out[:live] = y.to(out.dtype)
    return {"y": out, "experts": chosen.int(), "gates": share}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "product":
        m, n, k = case["rows"], case["n"], case["k"]
        blocks = -(-n // BLOCK) * -(-k // BLOCK)
        return {"bytes": 2.0 * m * k + 1.0 * n * k + blocks + (4.0 if case["fp32"] else 2.0) * m * n, "flops": 2.0 * m * n * k}
    d, ff, experts, top_k = case["d"], case["ff"], case["experts"], case["top_k"]
    live = case["rows"] - case["idle"]
    active = experts * (1.0 - (1.0 - top_k / experts) ** live)  # chosen by at least one row, where rows choose at random
    return {"bytes": active * 3.0 * d * ff * (1 if case["scaled"] else 2) + 2.0 * experts * d + 4.0 * live * d + 8.0 * live * top_k,
            "flops": 2.0 * live * (3.0 * top_k * d * ff + experts * d)}


# --------------------------------------------------------------------------- the same in 64 bits, written apart
def _e4m3_values():
    """The 127 magnitudes of e4m3, in the order of their bit patterns."""
    return torch.tensor([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)], dtype=torch.float64, device=DEVICE)


def _exact_blocks(x, tall):
    """What x [n][k] becomes in blocks of 128 columns and 128 rows (`tall`) or one row: values in 64 bits."""
    x = x.double()
    table = _e4m3_values()
    middle = (table[1:] + table[:-1]) / 2
    powers = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64, device=DEVICE)
    out = torch.empty_like(x)
    for r0 in range(0, x.shape[0], BLOCK):
        part = x[r0:r0 + BLOCK]
        most = torch.stack([c.abs().amax(-1) for c in part.split(BLOCK, dim=1)], 1)  # [rows][blocks]
        if tall:
            most = most.amax(0, keepdim=True).expand(part.shape[0], -1)
        power = torch.where(most > 0, powers[torch.bucketize(most / LARGEST, powers)], 1.0)  # the smallest that is not below
        power = power.repeat_interleave(BLOCK, 1)[:, :x.shape[1]]
        v = (part / power).contiguous()
        below = torch.bucketize(v.abs(), middle)                         # a value in the middle goes down ...
        tie = v.abs() == middle[below.clamp(max=125)]
        code = torch.where(tie & (below % 2 == 1), below + 1, below)     # ... unless the one above has the even pattern
        out[r0:r0 + BLOCK] = torch.sign(v) * table[code] * power
    return out


def exact(case, seed):
    if case["op"] == "product":
        x = _exact_blocks(_rows(case, case["k"], seed), False)
        w = _exact_blocks(_weights(case, case["n"], case["k"], seed), True)
        return x @ w.T
    live = case["rows"] - case["idle"]
    x = _rows(case, case["d"], seed)[:live].double()
    logits = x @ _router(case, seed).double().T
    share = torch.softmax(logits, -1)
    chosen = torch.argsort(logits, dim=-1, descending=True, stable=True)[:, :case["top_k"]]
    gates = torch.gather(share, 1, chosen)
    if case["renormalise"]:
        gates = gates / gates.sum(1, keepdim=True)
    y = torch.zeros((case["rows"], case["d"]), dtype=torch.float64, device=DEVICE)
    for e in sorted(set(chosen.flatten().tolist())):
        gate, up, down = (_exact_blocks(w, True) if case["scaled"] else w.double() for w in _expert(case, e, seed))
        mine = (chosen == e)
        rows = mine.any(1)
        weight = (gates * mine).sum(1)[rows]
        part = x[rows]
        a = part @ gate.T
        y[:live][rows] += weight[:, None] * ((a * torch.sigmoid(a) * (part @ up.T)) @ down.T)
    return {"y": y, "experts": chosen.int(), "gates": gates}
