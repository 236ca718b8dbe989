"""Reference of the 8-bit matrices, their products and the layer of experts, in 64 bits (not collected by pytest)."""
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # of a rounding, relative to the value
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}      # and near zero
E4M3 = torch.tensor([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)], dtype=torch.float64)
POWERS = torch.tensor([2.0 ** e for e in range(-110, 121)], dtype=torch.float64)


def e4m3(v):
    """|v| <= 448 (or NaN) -> the nearest e4m3 value, ties to the even pattern; infinities are NaN."""
    middle = (E4M3[1:] + E4M3[:-1]) / 2
    a = torch.nan_to_num(v.abs(), nan=0.0, posinf=0.0)
    below = torch.bucketize(a, middle)
    tie = a == middle[below.clamp(max=125)]
    code = torch.where(tie & (below % 2 == 1), below + 1, below)
    return torch.where(torch.isfinite(v), torch.sign(v) * E4M3[code], torch.nan)


def blocks(x, tall):
    """x [n][k] (any type, on any device) as it is held in blocks of 128 columns and 128 rows (`tall`) or one row: 64 bits, on the CPU."""
    x = x.detach().cpu().double()
    n, k = x.shape
    out = torch.empty_like(x)
    for r0 in range(0, n, 128):
        for c0 in range(0, k, 128):
            part = x[r0:r0 + 128, c0:c0 + 128]
            most = torch.nan_to_num(part.abs(), nan=0.0, posinf=0.0)
            most = most.amax() if tall else most.amax(1, keepdim=True)
            scale = POWERS[torch.bucketize(most / 448.0, POWERS).clamp(max=len(POWERS) - 1)]
            out[r0:r0 + 128, c0:c0 + 128] = e4m3(part / scale) * scale
    return out


def sum_steps(k):
    """Roundings of an fp32 sum of k products, each of at most 2^-24 of the sum of their magnitudes: an instruction adds 32 products to what is there and
    rounds in at most four places; sixteen more for joining the parts of several waves."""
    return (k / 8 + 16) * 2.0 ** -24


def rounded(value, error, dtype):
    """Bound on the distance of a result in `dtype` from `value`, where what was rounded is within `error` of it."""
    return error + (value.abs() + error) * HALF_STEP[dtype] + SMALLEST[dtype]


def product(x, w_values, dtype, eight_bit):
    """(result, bound) of rows x with a matrix whose held values are w_values.  eight_bit: by the 8-bit instruction, which cuts eight consecutive products
    to units of 2^-13 of the largest one's power of two before it adds them up: 2^-10 of a product as large as the group's largest factors make one."""
    xv = blocks(x, False)
    value, size = xv @ w_values.T, xv.abs() @ w_values.abs().T
    error = size * sum_steps(x.shape[1])
    if eight_bit:
        largest = [v.abs().reshape(v.shape[0], -1, 8).amax(2) for v in (xv, w_values)]
        error = error + largest[0] @ largest[1].T * 2.0 ** -10
    return value, rounded(value, error, dtype)


def close(got, want, bound, what=""):
    got = got.detach().cpu().double()
    bad = ~((got - want).abs() <= bound) & ~(torch.isnan(got) & torch.isnan(want)) & ~(got == want)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i].item()} instead of {want[i].item()} +- {bound[i].item()}")


def choose(x, router, top_k, renormalise):
    """(experts, shares) of every row in 64 bits; NaN logits count as the least, equal ones in ascending order."""
    logits = x.detach().cpu().double() @ router.detach().cpu().double().T
    order = torch.argsort(torch.where(torch.isnan(logits), -torch.inf, logits), dim=1, descending=True, stable=True)[:, :top_k]
    picked = torch.gather(logits, 1, order)
    p = torch.exp(picked - picked[:, :1])
    return order, p / (p.sum(1, keepdim=True) if renormalise else torch.exp(logits - picked[:, :1]).sum(1, keepdim=True))


def experts(x, matrices, chosen, share):
    """(result, bound in front of the last rounding) of the layer; matrices: per expert the held values of gate, up and down in 64 bits."""
    x = x.detach().cpu().double()
    y = torch.zeros((x.shape[0], x.shape[1]), dtype=torch.float64)
    bound = torch.zeros_like(y)
    d = x.shape[1]
    for e, (gate, up, down) in enumerate(matrices):
        row, place = torch.nonzero(chosen == e, as_tuple=True)
        if len(row) == 0:
            continue
        part, g = x[row], share[row, place][:, None]
        a, b = part @ gate.T, part @ up.T
        ea, eb = ((part.abs() @ m.abs().T) * sum_steps(d) for m in (gate, up))
        sig = torch.sigmoid(a)
        h = a * sig * b * g
        # silu's slope is at most 1.1; exp, division and three products in fp32: a handful of roundings; the pair of bf16 keeps 2^-17 of h, and the
        # product of the two small halves, which is left out in fp16, is below 2^-17 of h too; bf16 has no normal values below 2^-126
        eh = g * (1.1 * ea * (b.abs() + eb) + (a * sig).abs() * eb) + h.abs() * (16 * 2.0 ** -24 + a.abs() * 2.0 ** -23 + 2.0 ** -16) + 2.0 ** -126
        ff = gate.shape[0]
        y[row] += h @ down.T
        bound[row] += eh @ down.abs().T + (h.abs() @ down.abs().T) * sum_steps(3 * ff * chosen.shape[1])
    return y, bound
