"""Oracle of the operators around a routed layer step, in float64 numpy: the residual norm with its 8-bit output, the
router with its balance loss and gradient, 4-bit weights and the layer on them.  Written from the formulas that
include/mlpmoe.h states; where the library fixes an fp32 or bf16 rounding (scales, codes) the same rounding is made here."""
import numpy as np

from .mlpmoe_oracle import branch_offsets, round_to_bf16, silu

E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126


def round_to_e4m3(a):
    """Nearest e4m3 value (ties to even), values beyond 448 to 448: steps of 2^-9 below 2^-6, else 2^(e - 3)."""
    a = np.clip(np.asarray(a, dtype=np.float64), -E4M3_MAX, E4M3_MAX)
    e = np.floor(np.log2(np.maximum(np.abs(a), 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    return np.rint(a / step) * step


def add_rmsnorm(x, r=None, gain=None, eps=1e-6):
    """(s, v): s = x + r, v = s / sqrt(mean(s^2) + eps) * gain."""
    s = np.asarray(x, dtype=np.float64)
    if r is not None:
        s = s + np.asarray(r, dtype=np.float64)
    v = s / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps)
    return s, v if gain is None else v * np.asarray(gain, dtype=np.float64)


def quantize_e4m3(v, group=0):
    """(codes, scales) of the rows of v, one scale per `group` columns (0: per row)."""
    n, d = v.shape
    group = group or d
    codes, scales = np.zeros_like(v), np.zeros((n, -(-d // group)))
    for i, lo in enumerate(range(0, d, group)):
        part = v[:, lo:lo + group]
        scales[:, i] = np.maximum(np.abs(part).max(axis=1) / E4M3_MAX, SCALE_MIN)
        codes[:, lo:lo + group] = round_to_e4m3(part / scales[:, i:i + 1])
    return codes, scales


def _eligible(logits, avail, valid):
    ok = ~np.isnan(logits) & (logits > -np.inf)
    if avail is not None:
        ok &= np.asarray(avail, dtype=bool)[None, :]
    if valid is not None:
        ok &= np.asarray(valid, dtype=bool)[:, None]
    return ok


def _probabilities(logits, ok):
    x = np.where(ok, np.minimum(np.where(ok, logits, 0.0), np.finfo(np.float32).max), -np.inf)
    top = np.max(x, axis=1, keepdims=True, initial=-np.inf)
    e = np.where(ok, np.exp(np.where(ok, x, 0.0) - np.where(np.isfinite(top), top, 0.0)), 0.0)
    return e / np.maximum(e.sum(axis=1, keepdims=True), 1e-300)


def route(logits, top_k, avail=None, valid=None):
    """dict(select, counts, prob, loss, p): the selection, the tokens per branch (and, last, the routed tokens), the mean
    probabilities and the balance loss.  Row by row, the largest first, ties to the lowest index."""
    logits = np.asarray(logits, dtype=np.float64)
    n, B = logits.shape
    ok = _eligible(logits, avail, valid)
    select = np.zeros((n, B), dtype=np.uint8)
    for t in range(n):
        order = sorted((b for b in range(B) if ok[t, b]), key=lambda b: (-logits[t, b], b))
        select[t, order[:top_k]] = 1
    p = _probabilities(logits, ok)
    routed = int(ok.any(axis=1).sum())
    counts = select.astype(np.int64).sum(axis=0)
    prob = p.sum(axis=0) / max(routed, 1)
    n_avail = B if avail is None else int(np.count_nonzero(avail))
    loss = float(n_avail * np.dot(counts, prob) / max(int(counts.sum()), 1))
    return dict(select=select, counts=np.append(counts, routed), prob=prob, loss=loss, p=p)


def route_grad(logits, counts, avail=None, valid=None, grad_loss=1.0):
    """(grad, size): d(grad_loss * loss) / d logits at constant counts, and the sum of the magnitudes of its two terms."""
    logits = np.asarray(logits, dtype=np.float64)
    p = _probabilities(logits, _eligible(logits, avail, valid))
    n_avail = logits.shape[1] if avail is None else int(np.count_nonzero(avail))
    f = counts[:-1] / max(int(counts[:-1].sum()), 1)
    scale = grad_loss * n_avail / max(int(counts[-1]), 1)
    mean = p @ f
    return scale * p * (f[None, :] - mean[:, None]), abs(scale) * p * (f[None, :] + mean[:, None])


def w4_quantize(W, group, asymmetric):
    """(codes uint8 [rows x cols], scales float32 [groups x rows] (bf16 values), zeros uint8 [groups x rows]) of an fp32 matrix."""
    W = np.asarray(W, dtype=np.float32)
    rows, cols = W.shape
    codes, scales, zeros = np.zeros((rows, cols), np.uint8), [], []

    def flushed(s):
        return np.where(s < np.float32(2.0 ** -126), np.float32(0), s)
    for lo in range(0, cols, group):
        w = W[:, lo:lo + group]
        if asymmetric:
            mn, mx = np.minimum(w.min(axis=1), np.float32(0)), np.maximum(w.max(axis=1), np.float32(0))
            s = flushed(round_to_bf16((mx - mn) / np.float32(15)).astype(np.float32))
            div = np.where(s > 0, s, np.float32(1))
            z = np.clip(np.rint(-mn / div), 0, 15)
        else:
            s = flushed(round_to_bf16(np.abs(w).max(axis=1) / np.float32(7)).astype(np.float32))
            div = np.where(s > 0, s, np.float32(1))
            z = np.full(rows, 8.0, np.float32)
        codes[:, lo:lo + group] = np.clip(np.rint(w / div[:, None]) + z[:, None], 0, 15)
        scales.append(s)
        zeros.append(z.astype(np.uint8))
    return codes, np.stack(scales), np.stack(zeros)


def w4_dequantize(codes, scales, zeros, group):
    """(code - zero) * scale, exact in float64."""
    cols = codes.shape[1]
    s = np.repeat(scales.astype(np.float64).T, group, axis=1)[:, :cols]
    z = np.repeat(zeros.astype(np.float64).T, group, axis=1)[:, :cols]
    return (codes.astype(np.float64) - z) * s


def w4_pack(codes, scales, zeros, pad=0):
    """(q, scale, zero) in the stored layout, scale as float32; the padding holds `pad` (codes, zeros) and NaN (scales)."""
    rows, cols = codes.shape
    q = np.full((rows, -(-cols // 32) * 32), pad, np.uint8)
    q[:, :cols] = codes
    n_g, rows16 = scales.shape[0], -(-rows // 16) * 16
    s = np.full((n_g, rows16), np.nan, np.float32)
    s[:, :rows] = scales
    z = np.full((n_g, rows16), pad, np.uint8)
    z[:, :rows] = zeros
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8), s, z


def w4_unpack(q, rows, cols):
    """Codes [rows x cols] of the stored bytes."""
    both = np.stack((q & 15, q >> 4), axis=2).reshape(rows, -1)
    return both[:, :cols]


def w4_layer_forward(x, Wg, Wu, Wd, d_b, alpha=None, select=None, compensate=True, residual=None):
    """y of the layer whose matrices (Wg, Wu [I x d], Wd [d x I]) the codes stand for, in float64, and what the error of
    an fp32 evaluation scales with: dict(y, gate, up, h, abs_gate, abs_up, coef) with abs_* the sums of magnitudes."""
    x = np.asarray(x, dtype=np.float64)
    off = branch_offsets(d_b)
    B = len(d_b)
    alpha = np.ones(B) if alpha is None else np.asarray(alpha, dtype=np.float64)
    on = np.broadcast_to(alpha != 0, (x.shape[0], B)).copy()
    coef = np.ones(x.shape[0])
    if select is not None:
        on &= np.asarray(select) != 0
        k = on.sum(axis=1)
        if compensate:
            coef = np.sqrt(np.count_nonzero(alpha) / np.maximum(k, 1))
    gate, up = x @ Wg.T, x @ Wu.T
    h = np.zeros_like(gate)
    for b in range(B):
        sl = slice(off[b], off[b + 1])
        h[:, sl] = np.where(on[:, b:b + 1], alpha[b] * silu(gate[:, sl]) * up[:, sl], 0.0)
    y = coef[:, None] * (h @ Wd.T)
    if residual is not None:
        y = y + np.asarray(residual, dtype=np.float64)
    neuron_on = np.repeat(on, np.asarray(d_b), axis=1)
    neuron_alpha = np.repeat(alpha, np.asarray(d_b))
    return dict(y=y, gate=gate, up=up, h=h, abs_gate=np.abs(x) @ np.abs(Wg).T, abs_up=np.abs(x) @ np.abs(Wu).T, coef=coef,
                on=neuron_on, alpha=neuron_alpha)
