"""float64 oracle of the operators of a training step around a routed layer: the sorted order of the tokens, rows moved to their
branches and summed back with the gradient, LayerNorm, the norms' gradient, and AdamW with moments in 8 bits.  Written from the
formulas; shares no code with the CUDA library."""
import numpy as np

from .operators_oracle import quantize_e4m3, round_to_e4m3

M32 = 0xFFFFFFFF


def sort_tokens(select, slots, align):
    """Branch by branch, tokens ascending; a token's first `slots` branches; -1 where there is nothing."""
    n, B = select.shape
    offsets, counts, row_token = np.zeros(B + 1, np.int64), np.zeros(B, np.int64), []
    taken = [[b for b in range(B) if select[t, b]][:slots] for t in range(n)]
    members = [[] for _ in range(B)]
    for t, branches in enumerate(taken):
        for b in branches:
            members[b].append(t)
    token_row, token_branch = np.full((n, slots), -1, np.int64), np.full((n, slots), -1, np.int64)
    filled = np.zeros(n, np.int64)
    for b in range(B):
        counts[b] = len(members[b])
        for t in members[b]:
            token_row[t, filled[t]], token_branch[t, filled[t]] = len(row_token), b
            filled[t] += 1
            row_token.append(t)
        row_token += [-1] * (-len(members[b]) % align)
        offsets[b + 1] = len(row_token)
    return {"offsets": offsets, "counts": counts, "row_token": np.array(row_token, np.int64), "token_row": token_row, "token_branch": token_branch}


def sort_tokens_of_many(select, slots, align):
    """sort_tokens, a branch at a time."""
    taken = select != 0
    place = np.cumsum(taken, axis=1, dtype=np.int16)
    taken &= place <= slots
    n, B = taken.shape
    counts = taken.sum(axis=0)
    offsets = np.concatenate(([0], np.cumsum(-(-counts // align) * align)))
    row_token = np.full(offsets[B], -1, np.int64)
    token_row, token_branch = np.full((n, slots), -1, np.int64), np.full((n, slots), -1, np.int64)
    for b in range(B):
        t = np.flatnonzero(taken[:, b])
        row = offsets[b] + np.arange(t.size)
        row_token[row] = t
        token_row[t, place[t, b] - 1], token_branch[t, place[t, b] - 1] = row, b
    return {"offsets": offsets, "counts": counts, "row_token": row_token, "token_row": token_row, "token_branch": token_branch}


def combine(rows, token_row, weight=None, residual=None):
    n, slots = token_row.shape
    y = np.zeros((n, rows.shape[1]))
    for t in range(n):
        for j in range(slots):
            if token_row[t, j] >= 0:
                y[t] += rows[token_row[t, j]] * (1.0 if weight is None else weight[t, j])
    return y if residual is None else residual + y


def combine_grad(grad_y, rows, token_row, weight=None):
    """(grad_rows, grad_weight); rows without a token have a gradient of 0."""
    n, slots = token_row.shape
    grad_rows, grad_weight = np.zeros(rows.shape), np.zeros((n, slots))
    for t in range(n):
        for j in range(slots):
            r = token_row[t, j]
            if r >= 0:
                grad_rows[r] = grad_y[t] * (1.0 if weight is None else weight[t, j])
                grad_weight[t, j] = np.dot(grad_y[t], rows[r])
    return grad_rows, grad_weight


def add_layernorm(x, r, gain, bias, eps=1e-5):
    """(s, v)"""
    s = x if r is None else x + r
    z = s - s.mean(axis=1, keepdims=True)
    v = z / np.sqrt((z * z).mean(axis=1, keepdims=True) + eps)
    return s, v * (1.0 if gain is None else gain) + (0.0 if bias is None else bias)


def norm_grad(layer, s, gain, grad_out, grad_s=None, eps=1e-5):
    """(grad_x, grad_gain, grad_bias)"""
    z = s - s.mean(axis=1, keepdims=True) if layer else s
    q = 1.0 / np.sqrt((z * z).mean(axis=1, keepdims=True) + eps)
    h = grad_out * (1.0 if gain is None else gain)
    dx = h - z * q * q * (h * z).mean(axis=1, keepdims=True)
    if layer:
        dx = dx - h.mean(axis=1, keepdims=True)
    dx = q * dx
    return dx if grad_s is None else grad_s + dx, (grad_out * z * q).sum(axis=0), grad_out.sum(axis=0)


def mix32(h):
    """The 32-bit finaliser of MurmurHash3, on Python integers or uint64 arrays."""
    h = h ^ (h >> 16)
    h = (h * 0x85EBCA6B) & M32
    h = h ^ (h >> 13)
    h = (h * 0xC2B2AE35) & M32
    return h ^ (h >> 16)


def adamw_noise(seed, step, tensor, n, first=0):
    """32 random bits for each of n elements of a tensor from `first` on (all in the same 2^32)."""
    key = mix32(mix32(mix32(seed & M32) ^ (seed >> 32)) ^ (step & M32))
    key = mix32(tensor ^ key)
    if first >> 32:
        key = mix32(key ^ (first >> 32))
    key = np.uint64(key)
    with np.errstate(over="ignore"):
        i = np.arange(n, dtype=np.uint64) + np.uint64(first & M32)
        h = (key + i * np.uint64(0x9E3779B1)) & np.uint64(M32)
        for shift, mul in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
            h = ((h ^ (h >> np.uint64(shift))) * np.uint64(mul)) & np.uint64(M32)
        return h ^ (h >> np.uint64(16))


def e4m3_up_or_down(a, noise16):
    """Values of 0 .. 448 in e4m3, up where the cut-off part and (noise16 + 1/2) / 2^16 of a step reach a whole step."""
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.minimum(np.floor(a / step + (noise16 + 0.5) * 2.0 ** -16) * step, 448.0)


def adamw_blocks(x, root, noise=None):
    """(codes as values, scales) of a moment in 8 bits, a scale per 128 elements."""
    n = x.size
    if noise is None:
        codes, scales = (part[0] for part in quantize_e4m3(x[None, :], 128))
    else:
        scales = np.array([max(np.abs(x[i:i + 128]).max() / 448.0, 2.0 ** -126) for i in range(0, n, 128)])
        y = np.minimum(np.abs(x) / np.repeat(scales, 128)[:n], 448.0)
        half = (noise >> np.uint64(16)) if root else (noise & np.uint64(0xFFFF))
        codes = np.copysign(e4m3_up_or_down(y, half.astype(np.float64)), x)
    if root:
        codes = np.where((x > 0) & (codes < 2.0 ** -9), 2.0 ** -9, codes)
    return codes, scales


def adamw_moments_fp32(g, m, m_scale, v, v_scale, beta1, beta2, grad_scale=1.0, noise=None):
    """(codes and scales of m, codes and scales of sqrt(v)) after a step, bit by bit: every product, sum and root rounded to fp32 in the
    order of the formulas, scale = max * fp32(1 / 448), value = x * fp32(1 / scale).  m, v: codes as values; everything finite."""
    f = np.float32
    g, m, v = np.asarray(g, f) * f(grad_scale), np.asarray(m, f), np.asarray(v, f)
    per = [np.repeat(np.asarray(s, f), 128)[:g.size] for s in (m_scale, v_scale)]
    m, v = m * per[0], np.square(v * per[1])
    m = f(beta1) * m + f(1.0 - beta1) * g
    v = f(beta2) * v + f(1.0 - beta2) * g * g
    out = []
    for x, shift, root in ((m, 0, False), (np.sqrt(v), 16, True)):
        top = np.array([np.abs(x[i:i + 128]).max() for i in range(0, x.size, 128)], f)
        scale = np.maximum(top * (f(1) / f(448)), f(2.0 ** -126))
        y = np.minimum(np.abs(x) * np.repeat(f(1) / scale, 128)[:x.size], f(448))
        if noise is None:
            codes = round_to_e4m3(y.astype(np.float64))
        else:
            base = np.where(y < f(2.0 ** -6), f(2.0 ** -6), f(0))
            extra = ((noise >> np.uint64(shift)) & np.uint64(0xFFFF)).astype(np.uint32) * np.uint32(16) | np.uint32(8)
            codes = (((y + base).view(np.uint32) + extra) & np.uint32(0xFFF00000)).view(f) - base
            codes = np.minimum(codes, f(448)).astype(np.float64)
        if root:
            codes = np.where((x > 0) & (codes < 2.0 ** -9), 2.0 ** -9, codes)
        out += [np.copysign(codes, x), scale.astype(np.float64)]
    return tuple(out)


def bf16_up_or_down(p, noise):
    """p, rounded to fp32, in bf16: away from zero where the 16 bits of mix32(noise ^ 0x9E3779B1) and the cut-off 16 bits make up a step."""
    extra = np.array([mix32(int(h) ^ 0x9E3779B1) & 0xFFFF for h in noise], np.uint64)
    bits = np.asarray(p, np.float64).astype(np.float32).view(np.uint32).astype(np.uint64)
    return ((bits + extra) & np.uint64(0xFFFF0000)).astype(np.uint32).view(np.float32).astype(np.float64)


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """(p, m, v) after the step, all in float64."""
    g = g * grad_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    p = p - lr * weight_decay * p - lr / (1.0 - beta1 ** step) * m / (np.sqrt(v / (1.0 - beta2 ** step)) + eps)
    return p, m, v

