"""Operators of a training step around a routed layer, as they are measured: each in a plain form (elementary torch operations
in 32 bits) and as the library's own call.

dispatch      tokens sorted by the branches that a router selected for them, and their rows copied to the branches
combine       y_t = residual_t + sum_j weight[t, j] * rows[row of the j-th branch of t]  (without weights: the dispatch's gradient)
combine_grad  gradients of the sum with respect to the rows and the weights
layernorm     s = x + r;  v = (s - mean(s)) / sqrt(var(s) + eps) * gain + bias;  v in fp32, bf16, or e4m3 with scales
norm_grad     gradient of the residual RMSNorm or LayerNorm with respect to s, and the sums over tokens for gain and bias
adamw         one AdamW step over many tensors, moments in fp32, or in e4m3 with a scale per 128 elements
"""
import math
import random

import torch

own = False

FP8_MAX = 448.0
TINY = 2.0 ** -126
BLOCK = 128
WORD = 0xFFFFFFFF
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


def listed():
    return [
        # a small batch of the Qwen-shaped layer: the smallest calls
        dict(name="dispatch 64x896", op="dispatch", n=64, B=16, k=4, d=896, dtype="bf16", group=0, align=1, valid=0),
        # a training batch of the Llama-shaped layer, 8 of 32 branches each, branches starting on tiles of 128 rows
        dict(name="dispatch 8192x4096", op="dispatch", n=8192, B=32, k=8, d=4096, dtype="bf16", group=0, align=128, valid=0),
        # the same layers' outputs summed into the residual stream; the small one with padded tokens
        dict(name="combine 64x896", op="combine", n=64, B=16, k=4, d=896, rows="bf16", y="fp32", residual="fp32", weight=1, align=1, valid=1),
        dict(name="combine 8192x4096", op="combine", n=8192, B=32, k=8, d=4096, rows="bf16", y="fp32", residual="fp32", weight=1, align=128, valid=0),
        # gradients: an odd width in fp32 on a padded batch, and the large batch
        dict(name="combine_grad 1000x901", op="combine_grad", n=1000, B=16, k=4, d=901, rows="fp32", y="fp32", weight=1, align=1, valid=1),
        dict(name="combine_grad 8192x4096", op="combine_grad", n=8192, B=32, k=8, d=4096, rows="bf16", y="bf16", weight=1, align=128, valid=0),
        # the norm before a layer: one sequence of an odd length, and a large batch with bf16 contributions
        dict(name="layernorm 77x896", op="layernorm", n=77, d=896, x="fp32", r="bf16", out="bf16", group=0, pad=0),
        dict(name="layernorm 16384x4096", op="layernorm", n=16384, d=4096, x="fp32", r="bf16", out="bf16", group=0, pad=0),
        # its gradient at the Qwen width (RMSNorm, one microbatch), and at the Llama width (LayerNorm) with the residual's gradient added
        dict(name="norm_grad 2048x896 rms", op="norm_grad", kind="rms", n=2048, d=896, s="fp32", g="bf16", res="fp32", out="fp32", bias=0, pad=0),
        dict(name="norm_grad 16384x4096", op="norm_grad", kind="layer", n=16384, d=4096, s="fp32", g="bf16", res="fp32", out="fp32", bias=1, pad=0),
        # routers and gains of a 24-layer Qwen-shaped stack: many small tensors, moments in fp32
        dict(name="adamw 24 routers", op="adamw", layers=24, d=896, B=16, inter=0, p="fp32", g="fp32", state="fp32", copy=0, stochastic=0),
        # one Llama-shaped layer in mixed precision: fp32 weights with a bf16 copy, bf16 gradients, moments in 8 bits
        dict(name="adamw llama 8 bit", op="adamw", layers=1, d=4096, B=32, inter=14336, p="fp32", g="bf16", state="e4m3", copy=1, stochastic=1),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dispatch", "combine", "combine_grad", "layernorm", "norm_grad", "adamw"])
    if op in ("dispatch", "combine", "combine_grad"):
        B = _spread(rng, 2, 128)
        k = rng.randint(1, min(B, 8))
        d = _spread(rng, 40, 8192)
        if rng.random() < 0.7:
            d = d // 8 * 8
        n = _spread(rng, 1, min(32768, (1 << 26) // (k * d)))
        c = dict(op=op, n=n, B=B, k=k, d=d, align=rng.choice([1, 1, 16, 128 if n * k >= 128 * B else 1]), valid=rng.randint(0, 1))
        if op == "dispatch":
            dtype = rng.choice(["bf16", "fp32", "e4m3"])
            return dict(c, dtype=dtype, group=rng.choice([0, 32, 128]) if dtype == "e4m3" else 0)
        c.update(rows=rng.choice(["bf16", "bf16", "fp32"]), y=rng.choice(["bf16", "fp32"]), weight=int(rng.random() < 0.75))
        return dict(c, residual=rng.choice(["none", "bf16", "fp32"])) if op == "combine" else dict(c, weight=1)
    if op in ("layernorm", "norm_grad"):
        d = _spread(rng, 33, 8192)
        if rng.random() < 0.7:
            d = max(8, d // 8 * 8)
        n = _spread(rng, 1, min(32768, (3 << 24) // d))
        c = dict(op=op, n=n, d=d, pad=rng.choice([0, 0, 8, 5]))
        if op == "layernorm":
            out = rng.choice(["fp32", "bf16", "bf16", "e4m3"])
            return dict(c, x=rng.choice(["fp32", "fp32", "bf16"]), r=rng.choice(["none", "bf16", "fp32"]), out=out,
                        group=rng.choice([0, 32, 128]) if out == "e4m3" else 0)
        kind = rng.choice(["rms", "layer"])
        return dict(c, kind=kind, s=rng.choice(["fp32", "fp32", "bf16"]), g=rng.choice(["fp32", "bf16"]), res=rng.choice(["none", "fp32", "bf16"]),
                    out=rng.choice(["fp32", "bf16"]), bias=rng.randint(0, 1) if kind == "layer" else 0)
    d, B = _spread(rng, 40, 4096), _spread(rng, 2, 64)
    inter = rng.choice([0, _spread(rng, 64, 7168)])
    p = rng.choice(["fp32", "fp32", "bf16"])
    layers = _spread(rng, 1, max(1, min(32, (1 << 26) // (d * (B + 1 + 3 * inter)))))
    return dict(op=op, layers=layers, d=d, B=B, inter=inter, p=p, g=rng.choice(["fp32", "bf16"]), state=rng.choice(["fp32", "e4m3"]),
                copy=rng.randint(0, 1) if p == "fp32" else 0, stochastic=rng.randint(0, 1))


def groups_of(cols, group):
    return -(-cols // group)


def capacity(case):
    """Rows that the sorted order can need: every token in k branches, every branch's end rounded up."""
    pairs = case["n"] * case["k"]
    return pairs + min(case["B"], pairs) * (case["align"] - 1)


def tensors_of(case):
    """(elements, weight decay) of a stack's tensors: router and gain of each layer, and its three matrices."""
    one = [(case["d"] * case["B"], 0.1), (case["d"], 0.0)] + ([(case["d"] * case["inter"], 0.1)] * 3 if case["inter"] else [])
    return one * case["layers"]


def sort_plain(select, slots, align, rows):
    """The sorted order: branch by branch, tokens ascending, a token's first `slots` branches; places of nothing are -1."""
    sel = select != 0
    sel = sel & (sel.cumsum(1) <= slots)
    n, B = sel.shape
    counts = sel.sum(0)
    ends = (-(-counts // align) * align).cumsum(0)
    offsets = torch.cat((torch.zeros_like(ends[:1]), ends))
    branch, token = sel.t().nonzero().unbind(1)
    first = counts.cumsum(0) - counts
    row = torch.arange(branch.numel(), device=sel.device) - first[branch] + offsets[branch]
    slot = (sel.cumsum(1) - 1)[token, branch]
    row_token = torch.full((rows,), -1, device=sel.device, dtype=torch.int32)
    row_token[row] = token.int()
    token_row = torch.full((n, slots), -1, device=sel.device, dtype=torch.int32)
    token_row[token, slot] = row.int()
    token_branch = torch.full((n, slots), -1, device=sel.device, dtype=torch.int32)
    token_branch[token, slot] = branch.int()
    return {"offsets": offsets.int(), "counts": counts.int(), "row_token": row_token, "token_row": token_row, "token_branch": token_branch}


def _mix(h):
    """The 32-bit finaliser of MurmurHash3."""
    h = h ^ (h >> 16)
    h = (h * 0x85EBCA6B) & WORD
    h = h ^ (h >> 13)
    h = (h * 0xC2B2AE35) & WORD
    return h ^ (h >> 16)


def _noise(seed, step, first, sizes, stride, device):
    """32 random bits for each element of the flat buffer, from (seed, step, tensor, element)."""
    key = _mix(_mix(_mix(seed & WORD) ^ (seed >> 32)) ^ step)
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=device), stride)
    at = torch.arange(tensor.numel(), device=device) - first[tensor]
    return _mix((_mix(tensor ^ key) + at * 0x9E3779B1) & WORD)


def _to_e4m3(x, noise, shift, root):
    """|x| <= 448 in e4m3: to nearest (noise None), or up with the probability of the rest; roots above zero stay above zero."""
    if noise is None:
        y = x.to(TYPES["e4m3"]).float()
    else:
        a = x.abs()
        small = a < 2.0 ** -6
        bits = torch.where(small, a + 2.0 ** -6, a).view(torch.int32)
        bits = (bits + ((((noise >> shift) & 0xFFFF) << 4) | 8).int()) & -0x100000
        y = bits.view(torch.float32)
        y = torch.where(small, y - 2.0 ** -6, y).clamp(max=FP8_MAX) * torch.sign(x)
    if root:
        y = torch.where((x > 0) & (y == 0), torch.full_like(y, 2.0 ** -9), y)
    return y.to(TYPES["e4m3"])


def _to_blocks(x, noise=None, shift=0, root=False):
    """(codes, scales) of a flat buffer, a scale for each 128 elements."""
    xb = x.view(-1, BLOCK)
    scale = (xb.abs().amax(1) / FP8_MAX).clamp(min=TINY)
    y = (xb * (1.0 / scale).unsqueeze(1)).clamp(-FP8_MAX, FP8_MAX).view(-1)
    return _to_e4m3(y, noise, shift, root), scale


def _from_blocks(codes, scales):
    return (codes.float().view(-1, BLOCK) * scales.unsqueeze(1)).view(-1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device=dev, generator=g) * std

    c = dict(case)
    op = c["op"]
    st = {"case": c}
    if op in ("dispatch", "combine", "combine_grad"):
        n, B, k, d = c["n"], c["B"], c["k"], c["d"]
        # a router that prefers some branches; padded tokens select nothing
        logits = normal(n, B) + normal(1, B, std=0.5)
        select = torch.zeros(n, B, device=dev, dtype=torch.uint8).scatter_(1, logits.topk(k, 1).indices, 1)
        if c["valid"]:
            select *= (torch.rand(n, 1, device=dev, generator=g) < 0.8).to(torch.uint8)
        st["select"] = select.contiguous()
        st["rows_max"] = capacity(c)
        plan = sort_plain(select, k, c["align"], st["rows_max"])
        if op == "dispatch":
            st["plan"] = {name: torch.full_like(t, -1) for name, t in plan.items()}
            x = normal(n, d)
            st["x_scale"] = st["row_scale"] = None
            if c["dtype"] == "e4m3":
                xg = c["group"] or d
                xp = torch.nn.functional.pad(x, (0, -d % xg)).view(n, -1, xg)
                st["x_scale"] = (xp.abs().amax(2) / FP8_MAX).clamp(min=TINY)
                x = (xp / st["x_scale"].unsqueeze(2)).view(n, -1)[:, :d]
                st["row_scale"] = torch.zeros(st["rows_max"], groups_of(d, xg), device=dev)
            st["x"] = x.to(TYPES[c["dtype"]]).contiguous()
            st["rows"] = torch.zeros(st["rows_max"], d, device=dev).to(TYPES[c["dtype"]])
            st["work"] = torch.empty(1 << 22, device=dev, dtype=torch.uint8)
            return st
        st["plan"] = plan
        st["rows"] = normal(st["rows_max"], d).to(TYPES[c["rows"]])
        st["weight"] = torch.softmax(torch.where(plan["token_row"] >= 0, normal(n, k), torch.full((n, k), -1e30, device=dev)), 1) if c["weight"] else None
        if op == "combine":
            st["residual"] = None if c["residual"] == "none" else normal(n, d, std=2.0).to(TYPES[c["residual"]])
            st["y"] = torch.empty(n, d, device=dev, dtype=TYPES[c["y"]])
        else:
            st["grad_y"] = normal(n, d).to(TYPES[c["y"]])
            st["grad_rows"] = torch.zeros_like(st["rows"])
            st["grad_weight"] = torch.empty(n, k, device=dev)
    elif op == "layernorm":
        n, d, pad = c["n"], c["d"], c["pad"]
        st["x"] = (normal(n, d + pad, std=2.0) + 0.5).to(TYPES[c["x"]])[:, :d]
        st["r"] = None if c["r"] == "none" else normal(n, d + pad).to(TYPES[c["r"]])[:, :d]
        st["gain"], st["bias"] = 1.0 + normal(d, std=0.1), normal(d, std=0.1)
        st["x_out"] = torch.empty(n, d, device=dev, dtype=TYPES[c["x"]])
        st["out"] = torch.empty(n, d, device=dev, dtype=TYPES[c["out"]])
        st["scales"] = torch.empty(n, groups_of(d, c["group"] or d), device=dev) if c["out"] == "e4m3" else None
    elif op == "norm_grad":
        n, d, pad = c["n"], c["d"], c["pad"]
        st["s"] = (normal(n, d + pad, std=2.0) + 0.5).to(TYPES[c["s"]])[:, :d]
        st["gain"] = 1.0 + normal(d, std=0.1)
        st["grad_out"] = normal(n, d + pad).to(TYPES[c["g"]])[:, :d]
        st["grad_s"] = None if c["res"] == "none" else normal(n, d + pad).to(TYPES[c["res"]])[:, :d]
        st["grad_x"] = torch.empty(n, d, device=dev, dtype=TYPES[c["out"]])
        st["grad_gain"] = torch.empty(d, device=dev)
        st["grad_bias"] = torch.empty(d, device=dev) if c["bias"] else None
        st["work"] = torch.empty((1 << 26) + 16 * n, device=dev, dtype=torch.uint8)
    else:
        sizes = [m for m, _ in tensors_of(c)]
        st["sizes"] = sizes
        stride = torch.tensor([groups_of(m, BLOCK) * BLOCK for m in sizes], device=dev)
        st["stride"], st["first"] = stride, stride.cumsum(0) - stride
        st["starts"] = st["first"].tolist()
        total = int(stride.sum())
        # every tensor starts on a block of one buffer; what is between them stays zero
        at = torch.arange(total, device=dev)
        tensor = torch.repeat_interleave(torch.arange(len(sizes), device=dev), stride)
        inside = (at - st["first"][tensor] < torch.tensor(sizes, device=dev)[tensor]).float()
        del at, tensor
        st["decay"] = torch.repeat_interleave(torch.tensor([w for _, w in tensors_of(c)], device=dev), stride)
        st["p"] = (normal(total, std=0.02) * inside).to(TYPES[c["p"]])
        st["g"] = (normal(total, std=1e-3) * inside).to(TYPES[c["g"]])
        m, root = normal(total, std=3e-4) * inside, (normal(total, std=1e-3).abs() + 2e-4) * inside
        del inside
        if c["state"] == "fp32":
            st["m"], st["v"], st["m_scale"], st["v_scale"] = m, root * root, None, None
        else:
            st["m"], st["m_scale"] = _to_blocks(m)
            st["v"], st["v_scale"] = _to_blocks(root, root=True)
        st["copy"] = st["p"].to(torch.bfloat16) if c["copy"] else None
        st["step"] = torch.tensor([7], device=dev)
        st["grad_scale"] = torch.tensor([0.5], device=dev)
        st["settings"] = dict(lr=5e-5, beta1=0.9, beta2=0.999, eps=1e-8, stochastic=bool(c["stochastic"]), seed=int(seed) * 0x9E3779B97F4A7C15 % (1 << 64))
    return st


def _dispatch_plain(st):
    c = st["case"]
    plan = sort_plain(st["select"], c["k"], c["align"], st["rows_max"])
    used = plan["row_token"] >= 0
    token = plan["row_token"].clamp(min=0).long()

    def rows_of(x):
        return torch.where(used.unsqueeze(1), x[token], torch.zeros((), device=x.device, dtype=x.dtype))

    x = st["x"].view(torch.uint8) if c["dtype"] == "e4m3" else st["x"]
    out = dict(plan, rows=rows_of(x).view(st["x"].dtype))
    if st["x_scale"] is not None:
        out["row_scale"] = rows_of(st["x_scale"])
    return out


def _picked(st):
    """The rows of each token's branches [n x k x d] in fp32, zeros where there is none."""
    row = st["plan"]["token_row"]
    return torch.where((row >= 0).unsqueeze(2), st["rows"][row.clamp(min=0).long()].float(), torch.zeros((), device=row.device))


def _combine_plain(st):
    p = _picked(st)
    if st["weight"] is not None:
        p = p * torch.where(st["plan"]["token_row"] >= 0, st["weight"], torch.zeros_like(st["weight"])).unsqueeze(2)
    y = p.sum(1)
    if st["residual"] is not None:
        y = st["residual"].float() + y
    return {"y": y.to(st["y"].dtype)}


def _combine_grad_plain(st):
    g, row = st["grad_y"].float(), st["plan"]["token_row"]
    token, slot = (row >= 0).nonzero().unbind(1)
    grad_rows = torch.zeros_like(st["rows"])
    w = st["weight"]
    grad_rows[row[token, slot].long()] = (w[token, slot].unsqueeze(1) * g[token]).to(grad_rows.dtype)
    return {"grad_rows": grad_rows, "grad_weight": (g.unsqueeze(1) * _picked(st)).sum(2)}


def _layernorm_plain(st):
    c = st["case"]
    s = st["x"].float()
    if st["r"] is not None:
        s = s + st["r"].float()
    z = s - s.mean(1, keepdim=True)
    v = z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-5) * st["gain"] + st["bias"]
    if c["out"] != "e4m3":
        return {"x_out": s.to(st["x"].dtype), "out": v.to(TYPES[c["out"]])}
    n, d, group = c["n"], c["d"], c["group"] or c["d"]
    vp = torch.nn.functional.pad(v, (0, -d % group)).view(n, -1, group)
    scales = (vp.abs().amax(2) / FP8_MAX).clamp(min=TINY)
    codes = (vp * (1.0 / scales).unsqueeze(2)).clamp(-FP8_MAX, FP8_MAX).view(n, -1)[:, :d].to(TYPES["e4m3"])
    return {"x_out": s.to(st["x"].dtype), "out": codes, "scales": scales}


def _norm_grad_plain(st):
    c = st["case"]
    s, dv = st["s"].float(), st["grad_out"].float()
    if c["kind"] == "layer":
        s = s - s.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-5)
    xh, h = s * r, dv * st["gain"]
    dx = h - xh * (h * xh).mean(1, keepdim=True)
    if c["kind"] == "layer":
        dx = dx - h.mean(1, keepdim=True)
    dx = r * dx
    if st["grad_s"] is not None:
        dx = st["grad_s"].float() + dx
    out = {"grad_x": dx.to(st["grad_x"].dtype), "grad_gain": (dv * xh).sum(0, dtype=torch.float64).float()}
    if c["bias"]:
        out["grad_bias"] = dv.sum(0, dtype=torch.float64).float()
    return out


def _adamw_plain(st):
    c, o = st["case"], st["settings"]
    step = 7
    g = st["g"].float() * st["grad_scale"]
    p = st["p"].float()
    eight = c["state"] == "e4m3"
    m = _from_blocks(st["m"], st["m_scale"]) if eight else st["m"]
    v = _from_blocks(st["v"], st["v_scale"]).square() if eight else st["v"]
    m = o["beta1"] * m + (1.0 - o["beta1"]) * g
    v = o["beta2"] * v + (1.0 - o["beta2"]) * g * g
    root = torch.sqrt(v)
    denom = root / math.sqrt(1.0 - o["beta2"] ** step) + o["eps"]
    p = p - o["lr"] * st["decay"] * p - o["lr"] / (1.0 - o["beta1"] ** step) * (m / denom)
    noise = _noise(o["seed"], step, st["first"], st["sizes"], st["stride"], p.device) if c["stochastic"] and (eight or c["p"] == "bf16") else None
    if c["p"] == "bf16" and noise is not None:
        up = (p.view(torch.int32) + (_mix(noise ^ 0x9E3779B1) & 0xFFFF).int()) & -0x10000
        st["p"].copy_(up.view(torch.float32))
    else:
        st["p"].copy_(p)
    if st["copy"] is not None:
        st["copy"].copy_(p)
    if eight:
        codes, scale = _to_blocks(m, noise, 0)
        st["m"].copy_(codes), st["m_scale"].copy_(scale)
        codes, scale = _to_blocks(root, noise, 16, True)
        st["v"].copy_(codes), st["v_scale"].copy_(scale)
    else:
        st["m"].copy_(m), st["v"].copy_(v)
    return _adamw_outputs(st)


def _adamw_outputs(st):
    return {name: st[name] for name in ("p", "m", "v", "m_scale", "v_scale", "copy") if st[name] is not None}


PLAIN = {"dispatch": _dispatch_plain, "combine": _combine_plain, "combine_grad": _combine_grad_plain, "layernorm": _layernorm_plain,
         "norm_grad": _norm_grad_plain, "adamw": _adamw_plain}


def _own(st):
    from paper_2511_21089_b200 import binding as lib
    kinds = {torch.bfloat16: lib.MLPMOE_BF16, torch.float32: lib.MLPMOE_FP32, torch.float8_e4m3fn: lib.MLPMOE_E4M3}
    c = st["case"]
    op = c["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "dispatch":
        plan = st["plan"]
        lib.mlpmoe_sort_tokens(st["select"], c["n"], c["B"], c["k"], plan["offsets"], plan["counts"], plan["row_token"], st["rows_max"],
                               plan["token_row"], st["work"], st["work"].numel(), align=c["align"], token_branch=plan["token_branch"], stream=stream)
        lib.mlpmoe_dispatch(st["x"], st["rows"], c["n"], c["d"], c["B"], c["k"], plan["offsets"], plan["counts"], plan["token_row"], st["rows_max"],
                            align=c["align"], dtype=kinds[st["x"].dtype], x_scale=st["x_scale"], row_scale=st["row_scale"], group=c["group"],
                            stream=stream)
        out = dict(plan, rows=st["rows"])
        return out if st["row_scale"] is None else dict(out, row_scale=st["row_scale"])
    if op == "combine":
        res = st["residual"]
        lib.mlpmoe_combine(st["rows"], st["rows_max"], st["plan"]["token_row"], c["k"], st["y"], c["n"], c["d"], weight=st["weight"], residual=res,
                           rows_dtype=kinds[st["rows"].dtype], residual_dtype=lib.MLPMOE_FP32 if res is None else kinds[res.dtype],
                           y_dtype=kinds[st["y"].dtype], stream=stream)
        return {"y": st["y"]}
    if op == "combine_grad":
        plan = st["plan"]
        lib.mlpmoe_combine_backward(st["grad_y"], st["rows"], st["rows_max"], plan["token_row"], c["k"], st["grad_rows"], st["grad_weight"], c["n"],
                                    c["d"], weight=st["weight"], B=c["B"], align=c["align"], offsets=plan["offsets"], counts=plan["counts"],
                                    grad_y_dtype=kinds[st["grad_y"].dtype], rows_dtype=kinds[st["rows"].dtype], stream=stream)
        return {"grad_rows": st["grad_rows"], "grad_weight": st["grad_weight"]}
    if op == "layernorm":
        x, r = st["x"], st["r"]
        lib.mlpmoe_add_layernorm(x, r, st["x_out"], st["out"], c["n"], c["d"], gain=st["gain"], bias=st["bias"], scales=st["scales"], group=c["group"],
                                 eps=1e-5, x_dtype=kinds[x.dtype], r_dtype=kinds[r.dtype] if r is not None else lib.MLPMOE_FP32,
                                 out_dtype=kinds[st["out"].dtype], x_stride=x.stride(0), r_stride=r.stride(0) if r is not None else 0, stream=stream)
        return {"x_out": st["x_out"], "out": st["out"]} if st["scales"] is None else {"x_out": st["x_out"], "out": st["out"], "scales": st["scales"]}
    if op == "norm_grad":
        s, g, res = st["s"], st["grad_out"], st["grad_s"]
        lib.mlpmoe_norm_backward(lib.MLPMOE_LAYERNORM if c["kind"] == "layer" else lib.MLPMOE_RMSNORM, s, g, st["grad_x"], c["n"], c["d"],
                                 st["work"], st["work"].numel(), gain=st["gain"], grad_s=res, grad_gain=st["grad_gain"], grad_bias=st["grad_bias"],
                                 eps=1e-5, s_dtype=kinds[s.dtype], grad_out_dtype=kinds[g.dtype], grad_x_dtype=kinds[st["grad_x"].dtype],
                                 grad_s_dtype=lib.MLPMOE_FP32 if res is None else kinds[res.dtype], s_stride=s.stride(0), grad_out_stride=g.stride(0),
                                 grad_s_stride=0 if res is None else res.stride(0), stream=stream)
        out = {"grad_x": st["grad_x"], "grad_gain": st["grad_gain"]}
        return out if st["grad_bias"] is None else dict(out, grad_bias=st["grad_bias"])
    if "list" not in st:  # the description of the tensors, which a program builds once
        decay = [w for _, w in tensors_of(c)]

        def part(name, i, unit=1):
            t = st[name]
            return None if t is None else t[st["starts"][i] // unit:][:groups_of(st["sizes"][i], unit)]

        st["list"] = lib.mlpmoe_adamw_tensors([
            dict(n=m, param=part("p", i), grad=part("g", i), m=part("m", i), v=part("v", i), m_scale=part("m_scale", i, BLOCK),
                 v_scale=part("v_scale", i, BLOCK), param_bf16=part("copy", i), weight_decay=decay[i], param_dtype=kinds[st["p"].dtype],
                 grad_dtype=kinds[st["g"].dtype], state_dtype=kinds[st["m"].dtype]) for i, m in enumerate(st["sizes"])])
    lib.mlpmoe_adamw(st["list"], step=st["step"], grad_scale=st["grad_scale"], stream=stream, **st["settings"])
    return _adamw_outputs(st)


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


def _size(name):
    return {"fp32": 4, "bf16": 2, "e4m3": 1, "none": 0}[name]


def work(case):
    op = case["op"]
    if op in ("dispatch", "combine", "combine_grad"):
        n, d, k = case["n"], case["d"], case["k"]
        pairs = n * k * (0.8 if case["valid"] else 1.0)
        if op == "dispatch":
            row = d * _size(case["dtype"]) + (4 * groups_of(d, case["group"] or d) if case["dtype"] == "e4m3" else 0)
            return {"bytes": n * case["B"] + (n + pairs) * row + 4 * pairs + 8 * n * k + 8 * case["B"], "flops": 0}
        size = _size(case["rows"])
        if op == "combine":
            return {"bytes": pairs * d * size + n * d * (_size(case["y"]) + _size(case["residual"])) + n * k * (4 + 4 * case["weight"]), "flops": 2 * pairs * d}
        return {"bytes": 2 * pairs * d * size + n * d * _size(case["y"]) + 12 * n * k, "flops": 3 * pairs * d}
    if op == "layernorm":
        n, d = case["n"], case["d"]
        b = n * d * (2 * _size(case["x"]) + _size(case["r"]) + _size(case["out"])) + 8 * d
        if case["out"] == "e4m3":
            b += 4 * n * groups_of(d, case["group"] or d)
        return {"bytes": b, "flops": 8 * n * d}
    if op == "norm_grad":
        n, d = case["n"], case["d"]
        return {"bytes": n * d * (_size(case["s"]) + _size(case["g"]) + _size(case["res"]) + _size(case["out"])) + 4 * d * (2 + case["bias"]), "flops": 14 * n * d}
    total = sum(m for m, _ in tensors_of(case))
    state = 16 if case["state"] == "fp32" else 4 + 16 / BLOCK
    return {"bytes": total * (2 * _size(case["p"]) + _size(case["g"]) + state + 2 * case["copy"]), "flops": 14 * total}


# The definitions in 64 bits.

def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "dispatch":
        plan = sort_plain(st["select"], case["k"], case["align"], st["rows_max"])
        rows = torch.zeros(st["rows_max"], case["d"], device=st["x"].device, dtype=torch.float64)
        at = (plan["row_token"] >= 0).nonzero().squeeze(1)
        rows[at] = st["x"].double()[plan["row_token"][at].long()]
        out = {name: None for name in plan} | {"rows": rows}
        if st["x_scale"] is not None:
            scale = torch.zeros(st["rows_max"], st["x_scale"].shape[1], device=rows.device, dtype=torch.float64)
            scale[at] = st["x_scale"].double()[plan["row_token"][at].long()]
            out["row_scale"] = scale
        return out
    if op in ("combine", "combine_grad"):
        row, w = st["plan"]["token_row"], st["weight"]
        n, k, d = case["n"], case["k"], case["d"]
        y = torch.zeros(n, d, device=row.device, dtype=torch.float64)
        if op == "combine":
            if st["residual"] is not None:
                y += st["residual"].double()
            for j in range(k):
                t = (row[:, j] >= 0).nonzero().squeeze(1)
                part = st["rows"][row[t, j].long()].double()
                y[t] += part if w is None else part * w[t, j].double()[:, None]
            return {"y": y}
        grad_rows = torch.zeros(st["rows"].shape, device=row.device, dtype=torch.float64)
        grad_w = torch.zeros(n, k, device=row.device, dtype=torch.float64)
        for j in range(k):
            t = (row[:, j] >= 0).nonzero().squeeze(1)
            at = row[t, j].long()
            gy = st["grad_y"][t].double()
            grad_rows[at] = gy * w[t, j].double()[:, None]
            grad_w[t, j] = torch.einsum("td,td->t", gy, st["rows"][at].double())
        return {"grad_rows": grad_rows, "grad_weight": grad_w}
    if op == "layernorm":
        s = st["x"].double()
        if st["r"] is not None:
            s = s + st["r"].double()
        var, mean = torch.var_mean(s, 1, correction=0, keepdim=True)
        v = (s - mean) * (var + 1e-5).pow(-0.5) * st["gain"].double() + st["bias"].double()
        if case["out"] != "e4m3":
            return {"x_out": s, "out": v}
        d, group = case["d"], case["group"] or case["d"]
        gi = torch.arange(d, device=v.device) // group
        scales = torch.zeros(case["n"], int(gi[-1]) + 1, device=v.device, dtype=torch.float64)
        scales = scales.scatter_reduce(1, gi.expand(case["n"], d), v.abs(), "amax", include_self=True).div(FP8_MAX).clamp(min=TINY)
        return {"x_out": s, "out": v / scales[:, gi], "scales": scales}
    if op == "norm_grad":
        s, dv, gain = st["s"].double(), st["grad_out"].double(), st["gain"].double()
        d = case["d"]
        centre = s.sum(1, keepdim=True) / d if case["kind"] == "layer" else 0.0
        sigma = (((s - centre) ** 2).sum(1, keepdim=True) / d + 1e-5).sqrt()
        xh = (s - centre) / sigma
        along = torch.einsum("td,td->t", dv * gain, xh)[:, None] / d
        dx = (dv * gain - along * xh) / sigma
        if case["kind"] == "layer":
            dx -= (dv @ gain)[:, None] / d / sigma
        if st["grad_s"] is not None:
            dx += st["grad_s"].double()
        out = {"grad_x": dx, "grad_gain": torch.einsum("td,td->d", dv, xh)}
        return out | {"grad_bias": dv.sum(0)} if case["bias"] else out
    o, t = st["settings"], 7
    g = st["g"].double() * 0.5
    m, v = st["m"].double(), st["v"].double()
    if case["state"] == "e4m3":
        m = m * st["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * st["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = m + (1 - o["beta1"]) * (g - m)
    v = v + (1 - o["beta2"]) * (g * g - v)
    p = st["p"].double()
    p = p * (1 - o["lr"] * st["decay"].double()) - o["lr"] * (m / (1 - o["beta1"] ** t)) / ((v / (1 - o["beta2"] ** t)).sqrt() + o["eps"])
    out = {"p": p, "m": m, "v": v}
    if case["state"] == "e4m3":
        for name, x in (("m", m), ("v", v.sqrt())):
            scale = x.view(-1, BLOCK).abs().amax(1).div(FP8_MAX).clamp(min=TINY)
            out[name], out[name + "_scale"] = x / scale.repeat_interleave(BLOCK), scale
    if case["copy"]:
        out["copy"] = p
    return out
