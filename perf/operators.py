"""Operators of a routed decode step, as they are measured: each in a plain form (elementary torch operations in
32 bits) and as the library's own call.

add_rmsnorm  s = x + r;  v = s / sqrt(mean(s^2) + eps) * gain;  v in fp32, bf16, or e4m3 with one scale per group
route        softmax over the available branches, the top k of each token, tokens per branch, balance loss
route_grad   gradient of the balance loss with respect to the logits
w4_quantize  a weight matrix to 4-bit codes with group scales, and back to bf16
w4_forward   the MLPMoE layer on 4-bit weights for a few tokens, with a branch selection per token
"""
import math
import random

import torch

own = False

FP8_MAX = 448.0
TINY = 2.0 ** -126
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


def listed():
    return [
        # one token of the Llama-8B-shaped stack: the residual's addition and the norm before the layer
        dict(name="norm 1x4096 bf16", op="add_rmsnorm", n=1, d=4096, x="fp32", r="bf16", out="bf16", group=0, pad=0),
        # a prefill of the same stack whose layer takes 8-bit activations with one scale per 128 columns
        dict(name="norm 16384x4096 e4m3", op="add_rmsnorm", n=16384, d=4096, x="fp32", r="bf16", out="e4m3", group=128, pad=0),
        # the router of a decode batch: 64 tokens, 64 branches
        dict(name="route 64x64", op="route", n=64, B=64, k=16, dtype="fp32", avail=0, valid=0, pad=0),
        # the routers of training batches: a large one with pruned branches, and a padded one; their gradients
        dict(name="route 131072x128", op="route", n=131072, B=128, k=16, dtype="fp32", avail=26, valid=0, pad=0),
        dict(name="route_grad 8192x32", op="route_grad", n=8192, B=32, k=8, dtype="bf16", avail=0, valid=1, pad=0),
        dict(name="route_grad 131072x128", op="route_grad", n=131072, B=128, k=16, dtype="fp32", avail=26, valid=0, pad=0),
        # weights of the Qwen-shaped and of the Llama-shaped layer to 4 bits
        dict(name="quantize 4864x896 g32", op="w4_quantize", rows=4864, cols=896, group=32, zero=0, dtype="fp32"),
        dict(name="quantize 14336x4096 g128", op="w4_quantize", rows=14336, cols=4096, group=128, zero=1, dtype="bf16"),
        # one token through the Qwen-shaped layer: the smallest layer call
        dict(name="w4 qwen n=1", op="w4_forward", n=1, d=896, inter=4864, B=16, k=0, group=64, zero=0, x="bf16", x_group=0, y="bf16", residual=0),
        # one token through the Llama-shaped layer, added to the residual stream
        dict(name="w4 llama n=1", op="w4_forward", n=1, d=4096, inter=14336, B=32, k=0, group=128, zero=1, x="bf16", x_group=0, y="fp32", residual=1),
        # a small batch with 8-bit activations, every token on 8 of 32 branches
        dict(name="w4 llama n=8 routed", op="w4_forward", n=8, d=4096, inter=14336, B=32, k=8, group=128, zero=0, x="e4m3", x_group=128, y="bf16", residual=0),
        # the largest decode batch
        dict(name="w4 llama n=64", op="w4_forward", n=64, d=4096, inter=14336, B=32, k=0, group=128, zero=1, x="bf16", x_group=0, y="bf16", residual=0),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["add_rmsnorm", "route", "route_grad", "w4_quantize", "w4_forward", "w4_forward"])
    if op == "add_rmsnorm":
        d = _spread(rng, 33, 8192)
        if rng.random() < 0.7:
            d = max(8, d // 8 * 8)
        n = _spread(rng, 1, min(32768, (1 << 26) // d))
        out = rng.choice(["fp32", "bf16", "e4m3", "e4m3"])
        return dict(op=op, n=n, d=d, x=rng.choice(["fp32", "fp32", "bf16"]), r=rng.choice(["none", "bf16", "fp32"]), out=out,
                    group=rng.choice([0, 32, 64, 128]) if out == "e4m3" else 0, pad=rng.choice([0, 0, 8, 5]))
    if op in ("route", "route_grad"):
        B = _spread(rng, 2, 128)
        return dict(op=op, n=_spread(rng, 1, 131072), B=B, k=rng.randint(1, min(B, 16)), dtype=rng.choice(["fp32", "bf16"]),
                    avail=rng.choice([0, B // 5]), valid=rng.randint(0, 1), pad=rng.choice([0, 0, 4, 3]))
    group = rng.choice([32, 64, 128])
    if op == "w4_quantize":
        return dict(op=op, rows=_spread(rng, 16, 8192), cols=_spread(rng, 40, 7168), group=group, zero=rng.randint(0, 1),
                    dtype=rng.choice(["bf16", "fp32"]))
    B = _spread(rng, 1, 64)
    x = rng.choice(["bf16", "bf16", "fp32", "e4m3"])
    return dict(op=op, n=_spread(rng, 1, 64), d=8 * _spread(rng, 8, 512), inter=16 * max(B, _spread(rng, 16, 800)), B=B,
                k=rng.choice([0, 0, max(1, B // 4)]), group=group, zero=rng.randint(0, 1), x=x, x_group=rng.choice([0, 128]) if x == "e4m3" else 0,
                y=rng.choice(["bf16", "fp32"]), residual=rng.randint(0, 1))


def branch_widths(inter, B):
    """Widths of B unequal branches of `inter` neurons, multiples of 16 (equal ones where B divides the units and B is a power of two)."""
    units = inter // 16
    if units % B == 0 and B & (B - 1) == 0:
        return [inter // B] * B
    cuts = sorted(random.Random(units * 131 + B).sample(range(1, units), B - 1))
    return [16 * (b - a) for a, b in zip([0] + cuts, cuts + [units])]


def groups_of(cols, group):
    return -(-cols // group)


def quantize_plain(w, group, asymmetric):
    """Codes [rows x cols] (uint8), scales and zeros [groups x rows] of an fp32 matrix: scale = bf16(range / 15) or bf16(amax / 7)."""
    rows, cols = w.shape
    n_g = groups_of(cols, group)
    wp = torch.nn.functional.pad(w, (0, n_g * group - cols)).view(rows, n_g, group)
    if asymmetric:
        lo, hi = wp.amin(2).clamp(max=0.0), wp.amax(2).clamp(min=0.0)
        s = ((hi - lo) / 15.0).to(torch.bfloat16).float()
        div = torch.where(s > 0, s, torch.ones_like(s))
        z = torch.round(-lo / div).clamp(0, 15)
    else:
        s = (wp.abs().amax(2) / 7.0).to(torch.bfloat16).float()
        div = torch.where(s > 0, s, torch.ones_like(s))
        z = torch.full_like(s, 8.0)
    q = (torch.round(wp / div.unsqueeze(2)) + z.unsqueeze(2)).clamp(0, 15).to(torch.uint8)
    return q.view(rows, n_g * group)[:, :cols], s.t().contiguous(), z.t().contiguous()


def pack4(q, s, z, asymmetric):
    """The stored form: codes two to a byte (low nibble first) with rows padded to 16 bytes, scales bf16 and zeros uint8
    [groups x rows padded to 16]."""
    rows, cols = q.shape
    q = torch.nn.functional.pad(q, (0, -cols % 32))
    packed = q[:, 0::2] | (q[:, 1::2] << 4)
    s = torch.nn.functional.pad(s, (0, -rows % 16)).to(torch.bfloat16)
    z = torch.nn.functional.pad(z, (0, -rows % 16)).to(torch.uint8)
    return packed.contiguous(), s.contiguous(), (z.contiguous() if asymmetric else None)


def unpack4(m, rows, cols, group):
    """The matrix in fp32 that (codes, scales, zeros) stand for."""
    packed, s, z = m
    q = torch.stack((packed & 15, packed >> 4), 2).view(rows, -1)[:, :cols].float()
    s = s[:, :rows].float().t().repeat_interleave(group, 1)[:, :cols]
    z = 8.0 if z is None else z[:, :rows].float().t().repeat_interleave(group, 1)[:, :cols]
    return (q - z) * s


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device=dev, generator=g) * std

    c = dict(case)
    op = c["op"]
    st = {"case": c}
    if op == "add_rmsnorm":
        n, d, pad = c["n"], c["d"], c["pad"]
        st["x"] = normal(n, d + pad, std=2.0).to(TYPES[c["x"]])[:, :d]
        st["r"] = None if c["r"] == "none" else normal(n, d + pad).to(TYPES[c["r"]])[:, :d]
        st["gain"] = 1.0 + normal(d, std=0.1)
        st["x_out"] = torch.empty(n, d, device=dev, dtype=TYPES[c["x"]])
        st["out"] = torch.empty(n, d, device=dev, dtype=TYPES[c["out"]])
        st["scales"] = torch.empty(n, groups_of(d, c["group"] or d), device=dev) if c["out"] == "e4m3" else None
    elif op in ("route", "route_grad"):
        n, B = c["n"], c["B"]
        # a router that prefers some branches, with values rounded coarsely enough that ties occur
        logits = normal(n, B + c["pad"]) + normal(1, B + c["pad"], std=0.5)
        st["logits"] = (torch.round(logits * 256) / 256).to(TYPES[c["dtype"]])[:, :B]
        st["avail"] = None
        if c["avail"]:
            st["avail"] = torch.ones(B, device=dev, dtype=torch.uint8)
            st["avail"][torch.randperm(B, device=dev, generator=g)[:c["avail"]]] = 0
        st["valid"] = (torch.rand(n, device=dev, generator=g) < 0.8).to(torch.uint8) if c["valid"] else None
        st["select"] = torch.empty(n, B, device=dev, dtype=torch.uint8)
        st["counts"] = torch.empty(B + 1, device=dev, dtype=torch.int32)
        st["prob"] = torch.empty(B, device=dev)
        st["loss"] = torch.empty(1, device=dev)
        st["work"] = torch.empty(1 << 20, device=dev, dtype=torch.uint8)
        if op == "route_grad":
            st["counts"] = _counts(*_select(st["logits"], c["k"], st["avail"], st["valid"])[:2])
            st["grad_loss"] = normal(1).abs() + 0.5
            st["grad"] = torch.empty(n, B, device=dev, dtype=TYPES[c["dtype"]])
    elif op == "w4_quantize":
        rows, cols, group = c["rows"], c["cols"], c["group"]
        st["W"] = normal(rows, cols, std=0.02).to(TYPES[c["dtype"]])
        st["q"] = torch.empty(rows, 16 * groups_of(cols, 32), device=dev, dtype=torch.uint8)
        st["scale"] = torch.empty(groups_of(cols, group), -(-rows // 16) * 16, device=dev, dtype=torch.bfloat16)
        st["zero"] = torch.empty(st["scale"].shape, device=dev, dtype=torch.uint8) if c["zero"] else None
        st["back"] = torch.empty(rows, cols, device=dev, dtype=torch.bfloat16)
    else:
        n, d, inter, B, group = c["n"], c["d"], c["inter"], c["B"], c["group"]
        st["mats"] = [pack4(*quantize_plain(normal(rows, cols, std=0.02), group, c["zero"]), c["zero"])
                      for rows, cols in ((inter, d), (inter, d), (d, inter))]
        st["d_b"] = branch_widths(inter, B)
        st["alpha"] = [1.0 + 0.4 * (((b * 7 + int(seed)) % 11) / 11.0 - 0.5) for b in range(B)]
        x = normal(n, d)
        st["x_scale"] = None
        if c["x"] == "e4m3":
            xg = c["x_group"] or d
            xp = torch.nn.functional.pad(x, (0, -d % xg)).view(n, -1, xg)
            st["x_scale"] = (xp.abs().amax(2) / FP8_MAX).clamp(min=TINY)
            x = (xp / st["x_scale"].unsqueeze(2)).view(n, -1)[:, :d]
        # rows of 8-bit activations start on 16 bytes
        st["x"] = torch.nn.functional.pad(x.to(TYPES[c["x"]]).view(torch.uint8).view(n, -1), (0, -d % 16)).view(TYPES[c["x"]])[:, :d] \
            if c["x"] == "e4m3" else x.to(TYPES[c["x"]])
        st["select"] = None
        if c["k"]:
            order = torch.rand(n, B, device=dev, generator=g).argsort(1)
            st["select"] = (order < c["k"]).to(torch.uint8).contiguous()
        st["residual"] = normal(n, d) if c["residual"] else None
        st["y"] = torch.empty(n, d, device=dev, dtype=TYPES[c["y"]])
        st["work"] = torch.empty(16 * n * (d + inter + 512) + (1 << 20), device=dev, dtype=torch.uint8)
    return st


def _select(logits, k, avail, valid):
    """(eligible, selected): the k largest eligible logits of each row, ties to the lowest index."""
    x = logits.float()
    ok = x > -math.inf
    if avail is not None:
        ok = ok & (avail != 0)
    if valid is not None:
        ok = ok & (valid != 0).unsqueeze(1)
    order = torch.where(ok, x, torch.full_like(x, -math.inf)).sort(dim=1, descending=True, stable=True).indices[:, :k]
    sel = torch.zeros(x.shape, device=x.device, dtype=torch.uint8).scatter_(1, order, 1)
    return ok, sel * ok


def _counts(ok, sel):
    return torch.cat((sel.sum(0, dtype=torch.int32), ok.any(1).sum(dtype=torch.int32).view(1)))


def _softmax(logits, ok):
    x = torch.where(ok, logits.float(), torch.full(logits.shape, -math.inf, device=logits.device))
    top = x.amax(1, keepdim=True)
    e = torch.where(ok, torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top))), torch.zeros_like(x))
    return e / e.sum(1, keepdim=True).clamp(min=1e-30)


def _route_plain(st):
    c = st["case"]
    ok, sel = _select(st["logits"], c["k"], st["avail"], st["valid"])
    counts = _counts(ok, sel)
    p = _softmax(st["logits"], ok)
    routed = counts[-1:].double().clamp(min=1)
    prob = p.sum(0, dtype=torch.float64) / routed
    f = counts[:-1].double() / counts[:-1].sum().clamp(min=1)
    n_avail = c["B"] - c["avail"]
    return {"select": sel, "counts": counts, "prob": prob.float(), "loss": (n_avail * (f * prob).sum()).float().view(1)}


def _route_grad_plain(st):
    c = st["case"]
    ok, _ = _select(st["logits"], 1, st["avail"], st["valid"])
    p = _softmax(st["logits"], ok)
    counts = st["counts"]
    f = counts[:-1].float() / counts[:-1].sum().clamp(min=1)
    n_avail = c["B"] - c["avail"]
    grad = st["grad_loss"] * n_avail / counts[-1].clamp(min=1) * p * (f - (p * f).sum(1, keepdim=True))
    return {"grad": grad.to(st["logits"].dtype)}


def _norm_plain(st):
    c = st["case"]
    s = st["x"].float()
    if st["r"] is not None:
        s = s + st["r"].float()
    v = s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-6) * st["gain"]
    if c["out"] != "e4m3":
        return {"x_out": s.to(st["x"].dtype), "out": v.to(TYPES[c["out"]])}
    n, d, group = c["n"], c["d"], c["group"] or c["d"]
    vp = torch.nn.functional.pad(v, (0, -d % group)).view(n, -1, group)
    scales = (vp.abs().amax(2) / FP8_MAX).clamp(min=TINY)
    codes = (vp * (1.0 / scales).unsqueeze(2)).clamp(-FP8_MAX, FP8_MAX).view(n, -1)[:, :d].to(torch.float8_e4m3fn)
    return {"x_out": s.to(st["x"].dtype), "out": codes, "scales": scales}


def _widths(st, device):
    return torch.repeat_interleave(torch.arange(len(st["d_b"]), device=device), torch.tensor(st["d_b"], device=device))


def _w4_plain(st):
    c = st["case"]
    n, d, inter, group = c["n"], c["d"], c["inter"], c["group"]
    x = st["x"].float()
    if st["x_scale"] is not None:
        x = x * st["x_scale"].repeat_interleave(c["x_group"] or d, 1)[:, :d]
    gate = x @ unpack4(st["mats"][0], inter, d, group).t()
    up = x @ unpack4(st["mats"][1], inter, d, group).t()
    branch = _widths(st, x.device)
    h = gate / (1.0 + torch.exp(-gate)) * up * torch.tensor(st["alpha"], device=x.device)[branch]
    coef = 1.0
    if st["select"] is not None:
        h = h * st["select"][:, branch].float()
        k = st["select"].sum(1, keepdim=True).float()
        coef = torch.sqrt(c["B"] / k.clamp(min=1))
    y = coef * (h @ unpack4(st["mats"][2], d, inter, group).t())
    if st["residual"] is not None:
        y = st["residual"] + y
    return {"y": y.to(TYPES[c["y"]])}


def _plain(st):
    op = st["case"]["op"]
    if op == "add_rmsnorm":
        return _norm_plain(st)
    if op == "route":
        return _route_plain(st)
    if op == "route_grad":
        return _route_grad_plain(st)
    if op == "w4_quantize":
        c = st["case"]
        q, s, z = quantize_plain(st["W"].float(), c["group"], c["zero"])
        m = pack4(q, s, z, c["zero"])
        return {"back": unpack4(m, c["rows"], c["cols"], c["group"]).to(torch.bfloat16), "scale": m[1][:, :c["rows"]]}
    return _w4_plain(st)


def _own(st):
    from paper_2511_21089_b200 import binding as lib
    kinds = {torch.bfloat16: lib.MLPMOE_BF16, torch.float32: lib.MLPMOE_FP32, torch.float8_e4m3fn: lib.MLPMOE_E4M3}
    c = st["case"]
    op = c["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "add_rmsnorm":
        x, r = st["x"], st["r"]
        lib.mlpmoe_add_rmsnorm(x, r, st["x_out"], st["out"], c["n"], c["d"], gain=st["gain"], scales=st["scales"], group=c["group"], eps=1e-6,
                               x_dtype=kinds[x.dtype], r_dtype=kinds[r.dtype] if r is not None else lib.MLPMOE_FP32, out_dtype=kinds[st["out"].dtype],
                               x_stride=x.stride(0), r_stride=r.stride(0) if r is not None else 0, stream=stream)
        return {"x_out": st["x_out"], "out": st["out"]} if st["scales"] is None else {"x_out": st["x_out"], "out": st["out"], "scales": st["scales"]}
    if op == "route":
        lib.mlpmoe_route(st["logits"], c["n"], c["B"], c["k"], st["select"], st["counts"], st["prob"], st["loss"], st["work"], st["work"].numel(),
                         dtype=kinds[st["logits"].dtype], stride=st["logits"].stride(0), avail=st["avail"], valid=st["valid"], stream=stream)
        return {"select": st["select"], "counts": st["counts"], "prob": st["prob"], "loss": st["loss"]}
    if op == "route_grad":
        lib.mlpmoe_route_backward(st["logits"], st["counts"], st["grad"], c["n"], c["B"], grad_loss=st["grad_loss"], dtype=kinds[st["logits"].dtype],
                                  stride=st["logits"].stride(0), avail=st["avail"], valid=st["valid"], stream=stream)
        return {"grad": st["grad"]}
    if op == "w4_quantize":
        rows, cols = c["rows"], c["cols"]
        lib.mlpmoe_w4_quantize(st["W"], rows, cols, c["group"], st["q"], st["scale"], st["zero"], dtype=kinds[st["W"].dtype], stream=stream)
        lib.mlpmoe_w4_dequantize(st["q"], st["scale"], st["zero"], rows, cols, c["group"], st["back"], dtype=lib.MLPMOE_BF16, stream=stream)
        return {"back": st["back"], "scale": st["scale"][:, :rows]}
    if "layer" not in st:  # the description of the layer's buffers, which a program builds once
        st["layer"] = lib.mlpmoe_w4_layer(c["d"], c["inter"], st["d_b"], c["group"], *st["mats"], alpha=st["alpha"])
    lib.mlpmoe_w4_forward(st["layer"], st["x"], st["y"], c["n"], st["work"], st["work"].numel(), x_dtype=kinds[st["x"].dtype],
                          x_stride=st["x"].stride(0), x_scale=st["x_scale"], x_group=c["x_group"], select=st["select"], compensate=True,
                          residual=st["residual"], y_dtype=kinds[st["y"].dtype], stream=stream)
    return {"y": st["y"]}


def run(state):
    return _own(state) if own else _plain(state)


def _size(name):
    return {"fp32": 4, "bf16": 2, "e4m3": 1, "none": 0}[name]


def _routed_neurons(case):
    """Neurons whose weights a call has to read: all of them, or, with k of B branches per token, the mean number that n tokens touch."""
    share = 1.0 if not case["k"] else 1.0 - (1.0 - case["k"] / case["B"]) ** case["n"]
    return share * case["inter"]


def work(case):
    op = case["op"]
    if op == "add_rmsnorm":
        n, d = case["n"], case["d"]
        b = n * d * (2 * _size(case["x"]) + _size(case["r"]) + _size(case["out"])) + 4 * d
        if case["out"] == "e4m3":
            b += 4 * n * groups_of(d, case["group"] or d)
        return {"bytes": b, "flops": 6 * n * d}
    if op == "route":
        n, B = case["n"], case["B"]
        return {"bytes": n * B * (_size(case["dtype"]) + 1) + n * case["valid"] + 8 * B, "flops": 8 * n * B}
    if op == "route_grad":
        n, B = case["n"], case["B"]
        return {"bytes": 2 * n * B * _size(case["dtype"]) + n * case["valid"] + 4 * B, "flops": 9 * n * B}
    if op == "w4_quantize":
        r, k = case["rows"], case["cols"]
        codes = r * k / 2 + r * groups_of(k, case["group"]) * (2 + case["zero"])
        return {"bytes": r * k * (_size(case["dtype"]) + 2) + 2 * codes, "flops": 6 * r * k}
    n, d, live = case["n"], case["d"], _routed_neurons(case)
    weights = 3 * d * live * (0.5 + (2 + case["zero"]) / case["group"])
    io = n * d * (_size(case["x"]) + _size(case["y"]) + 4 * case["residual"])
    pairs = n * case["inter"] * (case["k"] / case["B"] if case["k"] else 1.0)
    return {"bytes": weights + io, "flops": 6 * d * pairs}


# The definitions in 64 bits.

def _exact_w4(m, rows, cols, group):
    packed, s, z = m
    j = torch.arange(cols, device=packed.device)
    q = (packed[:, j // 2].to(torch.int64) >> (4 * (j % 2))) & 15
    gi = j // group
    zero = 8 if z is None else z[gi][:, :rows].t().to(torch.int64)
    return (q - zero).double() * s[gi][:, :rows].t().double()


def _exact_probs(st):
    x = st["logits"].double()
    ok = torch.isfinite(x)
    if st["avail"] is not None:
        ok &= st["avail"].bool()[None, :]
    if st["valid"] is not None:
        ok &= st["valid"].bool()[:, None]
    x = x.masked_fill(~ok, -math.inf)
    z = torch.logsumexp(x, 1, keepdim=True)
    return torch.exp(x - z.masked_fill(~torch.isfinite(z), 0.0)).masked_fill(~ok, 0.0), ok


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "add_rmsnorm":
        s = st["x"].double()
        if st["r"] is not None:
            s = s + st["r"].double()
        v = s * (s.pow(2).sum(1, keepdim=True) / case["d"] + 1e-6).pow(-0.5) * st["gain"].double()
        if case["out"] != "e4m3":
            return {"x_out": s, "out": v}
        d, group = case["d"], case["group"] or case["d"]
        gi = torch.arange(d, device=v.device) // group
        scales = torch.zeros(case["n"], int(gi[-1]) + 1, device=v.device, dtype=torch.float64)
        scales = scales.scatter_reduce(1, gi.expand(case["n"], d), v.abs(), "amax", include_self=True).div(FP8_MAX).clamp(min=TINY)
        w = (v / scales[:, gi]).clamp(-FP8_MAX, FP8_MAX)
        # e4m3: 4 significant bits down to 2^-6, steps of 2^-9 below
        step = torch.exp2(torch.floor(torch.log2(w.abs().clamp(min=2.0 ** -6))) - 3)
        return {"x_out": s, "out": torch.round(w / step) * step, "scales": scales}
    if op == "route":
        p, ok = _exact_probs(st)
        _, sel = _select(st["logits"], case["k"], st["avail"], st["valid"])
        cnt = sel.double().sum(0)
        routed = ok.any(1).double().sum().clamp(min=1)
        prob = p.sum(0) / routed
        loss = (case["B"] - case["avail"]) * torch.dot(cnt / cnt.sum().clamp(min=1), prob)
        return {"select": None, "counts": None, "prob": prob, "loss": loss.view(1)}
    if op == "route_grad":
        p, _ = _exact_probs(st)
        cnt = st["counts"].double()
        f = cnt[:-1] / cnt[:-1].sum().clamp(min=1)
        scale = st["grad_loss"].double() * (case["B"] - case["avail"]) / cnt[-1].clamp(min=1)
        return {"grad": scale * (p * f - p * (p @ f)[:, None])}
    if op == "w4_quantize":
        w = st["W"].double()
        rows, cols, group = case["rows"], case["cols"], case["group"]
        gi = torch.arange(cols, device=w.device) // group
        idx, n_g = gi.expand(rows, cols), int(gi[-1]) + 1
        zeros = torch.zeros(rows, n_g, device=w.device, dtype=torch.float64)
        if case["zero"]:
            lo, hi = zeros.scatter_reduce(1, idx, w, "amin"), zeros.scatter_reduce(1, idx, w, "amax")
            s = ((hi - lo) / 15).to(torch.bfloat16).double()
            z = torch.round(-lo / s.masked_fill(s == 0, 1.0)).clamp(0, 15)[:, gi]
        else:
            s = (zeros.scatter_reduce(1, idx, w.abs(), "amax") / 7).to(torch.bfloat16).double()
            z = 8.0
        q = (torch.round(w / s.masked_fill(s == 0, 1.0)[:, gi]) + z).clamp(0, 15)
        return {"back": (q - z) * s[:, gi], "scale": s.t()}
    d, inter, group = case["d"], case["inter"], case["group"]
    x = st["x"].double()
    if st["x_scale"] is not None:
        x = x * st["x_scale"].double()[:, torch.arange(d, device=x.device) // (case["x_group"] or d)]
    y, lo = torch.zeros(case["n"], d, device=x.device, dtype=torch.float64), 0
    up = x @ _exact_w4(st["mats"][1], inter, d, group).t()
    h = torch.nn.functional.silu(x @ _exact_w4(st["mats"][0], inter, d, group).t()) * up
    down = _exact_w4(st["mats"][2], d, inter, group)
    for b, width in enumerate(st["d_b"]):
        part = st["alpha"][b] * (h[:, lo:lo + width] @ down[:, lo:lo + width].t())
        y += part if st["select"] is None else part * st["select"][:, b:b + 1].double()
        lo += width
    if st["select"] is not None:
        y *= (case["B"] / st["select"].double().sum(1, keepdim=True).clamp(min=1)).sqrt()
    return {"y": y if st["residual"] is None else st["residual"].double() + y}
