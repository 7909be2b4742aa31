"""Cases for the operators of a gated network trained on a buffer: the gated feed-forward block (forward, and forward
with its backward pass), the softmax loss with its gradient, and the AdamW step over all tensors of the model.

Each case has an entry "op": "ffn", "ffn_train", "residual" or "adamw".  `run` computes the operator with elementary
torch operations where `own` is false, and calls the library where it is true.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
ACTIVATIONS = ("silu", "gelu", "relu", "sigmoid")   # in the library's numbering: 0, 1, 2, 3
BLOCK = 256                                         # elements that share a scale where the moments are held in 8 bits
MASK32 = 0xFFFFFFFF


def listed():
    return [
        # ---- the block without its gradient: rows x inputs -> hidden -> outputs
        # one row at a time: a request that is answered as it comes
        dict(name="ffn one row", op="ffn", rows=1, inputs=4096, hidden=11008, outputs=4096, type="bf16", act="silu", extra=0),
        # a handful of requests together, in fp16
        dict(name="ffn few rows", op="ffn", rows=13, inputs=2048, hidden=5632, outputs=2048, type="fp16", act="gelu", extra=0),
        # a buffer's rows scored in one call
        dict(name="ffn many rows", op="ffn", rows=4096, inputs=4096, hidden=11008, outputs=4096, type="bf16", act="silu", extra=0),
        # ---- the block in training: forward, then the gradients of the rows and of the three weights
        # a mini-batch of 1,000 rows of 512 extracted features, two classes
        dict(name="train features", op="ffn_train", rows=1000, inputs=512, hidden=1024, outputs=2, type="bf16", act="sigmoid", extra=0),
        # odd widths (500 predictors, as in the simulated sample) and rows that are a slice of a wider buffer
        dict(name="train odd widths", op="ffn_train", rows=777, inputs=500, hidden=1371, outputs=500, type="fp16", act="gelu", extra=12),
        # a wide block and a large mini-batch
        dict(name="train large", op="ffn_train", rows=8192, inputs=4096, hidden=11008, outputs=4096, type="bf16", act="silu", extra=0),
        # ---- softmax loss with its gradient
        # the mini-batch of a ten-class job
        dict(name="residual ten classes", op="residual", rows=256, classes=10, type="fp32", skipped=0),
        # many classes, an odd number of them, some rows without a label
        dict(name="residual many classes", op="residual", rows=8191, classes=50257, type="bf16", skipped=40),
        # ---- AdamW over all tensors of a stack of blocks (three weights and one vector each) with a head
        # the smallest model: latency of one call
        dict(name="adamw small", op="adamw", blocks=1, width=200, hidden=64, classes=10, param="fp32", grad="fp32", bits=32, master=False, clip=0.0),
        # many tensors of middling size, clipped by the norm of all gradients
        dict(name="adamw many clipped", op="adamw", blocks=48, width=512, hidden=1371, classes=10, param="fp32", grad="fp32", bits=32, master=False, clip=1.0),
        # bf16 weights with fp32 copies, fp32 moments
        dict(name="adamw copies", op="adamw", blocks=2, width=4096, hidden=11008, classes=1000, param="bf16", grad="bf16", bits=32, master=True, clip=0.0),
        # bf16 weights alone, moments in 8 bits: as little memory per weight as it gets
        dict(name="adamw 8 bits", op="adamw", blocks=2, width=4096, hidden=11008, classes=1000, param="bf16", grad="bf16", bits=8, master=False, clip=0.0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["ffn", "ffn", "ffn_train", "ffn_train", "residual", "adamw", "adamw"])
    if op in ("ffn", "ffn_train"):
        rows, most = _log(rng, 1, 4096), 4096
        inputs, hidden, outputs = _log(rng, 16, most), _log(rng, 16, 8192), _log(rng, 2, most)
        if rng.random() < 0.6:  # most models have widths of a multiple of eight
            inputs, hidden, outputs = -(-inputs // 8) * 8, -(-hidden // 8) * 8, -(-outputs // 8) * 8
        return dict(op=op, rows=rows, inputs=inputs, hidden=hidden, outputs=outputs, type=rng.choice(["bf16", "fp16"]),
                    act=rng.choice(ACTIVATIONS), extra=rng.choice([0, 0, 1, 8, 24]))
    if op == "residual":
        classes = _log(rng, 2, 130_000)
        rows = _log(rng, 1, min(16_384, 200_000_000 // classes))
        return dict(op=op, rows=rows, classes=classes, type=rng.choice(["bf16", "fp16", "fp32"]), skipped=rng.choice([0, rows // 5]))
    param = rng.choice(["fp32", "bf16", "fp16"])
    master = param == "fp16" or (param == "bf16" and rng.random() < 0.5)
    return dict(op=op, blocks=_log(rng, 1, 64), width=_log(rng, 8, 1024), hidden=_log(rng, 8, 2048), classes=_log(rng, 2, 2048),
                param=param, grad=rng.choice([param, "fp32"]), bits=rng.choice([32, 8]), master=master, clip=rng.choice([0.0, 0.5]))


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def sizes_of(case):
    """Element counts of the model's tensors: w_gate, w_up, w_down and a vector per block, then the head."""
    w, h = case["width"], case["hidden"]
    return [w * h, w * h, h * w, w] * case["blocks"] + [w * case["classes"]]


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case)
    if case["op"] in ("ffn", "ffn_train"):
        t = TYPES[case["type"]]
        n, d, f, c = case["rows"], case["inputs"], case["hidden"], case["outputs"]
        s["x"] = _normal(gen, (n, d + case["extra"]), t)[:, :d]       # rows of a wider buffer where extra > 0
        s["w_gate"] = _normal(gen, (d, f), t, d ** -0.5)
        s["w_up"] = _normal(gen, (d, f), t, d ** -0.5)
        s["w_down"] = _normal(gen, (f, c), t, f ** -0.5)
        if case["op"] == "ffn_train":
            s["dy"] = _normal(gen, (n, c), t, 0.1)
    elif case["op"] == "residual":
        n, c = case["rows"], case["classes"]
        s["logits"] = _normal(gen, (n, c), TYPES[case["type"]], 3.0)
        s["y"] = torch.randint(0, c, (n,), generator=gen, device="cuda", dtype=torch.int32)
        s["y"][:case["skipped"]] = -1
    else:
        sizes = sizes_of(case)
        padded = [-(-k // BLOCK) * BLOCK for k in sizes]              # every tensor is a piece of one flat buffer
        starts = [0]
        for k in padded:
            starts.append(starts[-1] + k)
        total = starts[-1]
        real = torch.zeros(total, dtype=torch.bool, device="cuda")
        for a, k in zip(starts, sizes):
            real[a:a + k] = True
        zero = lambda x: torch.where(real, x, torch.zeros((), dtype=x.dtype, device="cuda"))  # noqa: E731
        gscale = 1024.0 if case["grad"] == "fp16" else 1.0            # fp16 gradients come multiplied by a loss scale
        flat = {"grads": zero(_normal(gen, total, TYPES[case["grad"]], 1e-2 * gscale))}
        # per-element spread of gradients over a few orders of magnitude, as the rows of a layer show it
        spread = torch.exp2(torch.randint(-6, 7, (total,), generator=gen, device="cuda").float())
        p = zero(_normal(gen, total, torch.float32, 0.05))
        m = zero(_normal(gen, total, torch.float32, 3e-3) * spread)
        v = zero((_normal(gen, total, torch.float32, 1e-2) * spread).square() + m.square() * 0.5)
        del spread
        flat["params"] = p.to(TYPES[case["param"]])
        if case["master"]:
            flat["masters"] = p
        if case["bits"] == 8:
            bits = torch.zeros(total, dtype=torch.int64, device="cuda")
            flat["m"], flat["m_scale"] = encode_m(m, bits)
            flat["v"], flat["v_scale"] = encode_v(v, bits)
        else:
            flat["m"], flat["v"] = m, v
        s["flat"] = flat
        per = {"m_scale": BLOCK, "v_scale": BLOCK}
        # the tensors as the program has them: views, one for each tensor of the model
        s["lists"] = {k: [x[a // per.get(k, 1):(a + (e if k not in per else -(-e // BLOCK) * BLOCK)) // per.get(k, 1)]
                          for a, e in zip(starts, sizes)] for k, x in flat.items()}
        s["decays"] = [0.0 if k == case["width"] else 0.1 for k in sizes]   # the vectors are not decayed
        s["control"] = torch.zeros(4, dtype=torch.int64, device="cuda")
        s["control"][0] = 20
        s["gscale"] = 1.0 / gscale
        lengths = torch.tensor(padded, device="cuda")
        s["index"] = torch.tensor(list(range(len(sizes))), device="cuda")
        s["starts"] = torch.tensor(starts[:-1], device="cuda")
        s["lengths"] = lengths
        s["seed"] = int(seed) * 7919 + 5
    return s


# ---------------------------------------------------------------- plain forms

def activate(act, g):
    """act(g) and act'(g)."""
    if act == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-g))
    if act == "sigmoid":
        return sig, sig * (1.0 - sig)
    return g * sig, sig * (1.0 + g * (1.0 - sig))


def plain_ffn(s):
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    t = s["x"].dtype
    g, u = x @ wg, x @ wu
    a, da = activate(s["act"], g)
    h = a * u
    y = (h @ wd).to(t)
    if s["op"] == "ffn":
        return {"y": y}
    dy = s["dy"].float()
    dh = dy @ wd.T
    dg, du = dh * u * da, dh * a
    return {"y": y, "dx": (dg @ wg.T + du @ wu.T).to(t), "dw_gate": (x.T @ dg).to(t), "dw_up": (x.T @ du).to(t),
            "dw_down": (h.T @ dy).to(t)}


def plain_residual(s):
    z, y = s["logits"].float(), s["y"].long()
    with_label = ((y >= 0) & (y < z.shape[1])).unsqueeze(1)
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    at = y.clamp(0, z.shape[1] - 1).unsqueeze(1)
    loss = torch.where(with_label, torch.log(total) + top - z.gather(1, at), torch.zeros_like(top)).squeeze(1)
    r = e / total
    r.scatter_add_(1, at, torch.full_like(top, -1.0))
    r = torch.where(with_label, r * (1.0 / z.shape[0]), torch.zeros_like(r))
    return {"residual": r.to(s["logits"].dtype), "loss": loss}


def mix(x):
    """The 32-bit mixing function of the random bits (int64 tensors or numbers that hold 32-bit values)."""
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & MASK32
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & MASK32
    return x ^ (x >> 16)


def block_exponent(x, least):
    """Biased exponent of the largest finite magnitude of each block of 256, at least `least`."""
    a = x.abs()
    a = torch.where(torch.isfinite(a), a, torch.zeros_like(a)).view(-1, BLOCK).amax(dim=1)
    return (a.view(torch.int32) >> 23).clamp(min=least)


def power_of_two(biased):
    return (biased << 23).view(torch.float32)


def encode_m(m, bits):
    """First moments in 8 bits (e4m3), rounded at random by the low 16 bits of `bits`: codes and block exponents."""
    s = block_exponent(m, 16)
    x = (m.view(-1, BLOCK) * power_of_two(261 - s).unsqueeze(1)).view(-1)
    a, r = x.abs(), (bits & 0xFFFF).to(torch.int32)
    code = torch.where(a >= 2.0 ** -6, ((a.view(torch.int32) - (120 << 23)) + (r << 4)) >> 20,
                       (a * 512.0 + r.float() * (1.0 / 65536.0)).floor().clamp(max=8.0).to(torch.int32))
    code = torch.where(torch.isfinite(x), code, torch.full_like(code, 0x7F))
    code = code | ((x.view(torch.int32) >> 24) & 0x80)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), s.to(torch.uint8)


def decode_m(codes, s):
    return (codes.float().view(-1, BLOCK) * power_of_two(s.to(torch.int32) - 7).unsqueeze(1)).view(-1)


def encode_v(v, bits):
    """Second moments in 8 bits (five exponent and three mantissa bits, no sign), rounded at random by bits 16 to 31."""
    s = block_exponent(v, 40)
    y = (v.view(torch.int32).view(-1, BLOCK) - ((s - 30) << 23).unsqueeze(1)).view(-1)
    r = (bits >> 16).to(torch.int32)
    code = torch.where(y >= 1 << 20, (y + (r << 4)) >> 20, torch.ones_like(y))
    code = torch.where(v == 0, torch.zeros_like(code), code)
    code = torch.where(torch.isfinite(v), code, torch.full_like(code, 255))
    return code.to(torch.uint8), s.to(torch.uint8)


def decode_v(codes, s):
    c = codes.to(torch.int32)
    exponent = (c >> 3).view(-1, BLOCK) + (s.to(torch.int32) - 30).unsqueeze(1)
    x = ((exponent.view(-1) << 23) | ((c & 7) << 20)).view(torch.float32)
    x = torch.where(c == 0, torch.zeros_like(x), x)
    return torch.where(c == 255, torch.full_like(x, float("nan")), x)


HYPER = dict(lr=1e-3, a=0.9, b=0.999, eps=1e-8)


def plain_adamw(s):
    f, (lr, a, b, eps) = s["flat"], HYPER.values()
    g = f["grads"].float()
    t = s["control"][0] + 1
    scale = torch.full((), s["gscale"], dtype=torch.float64, device=g.device)
    fine = torch.ones((), dtype=torch.bool, device=g.device)
    if s["clip"] > 0:
        norm = f["grads"].double().square().sum().sqrt() * s["gscale"]
        fine = torch.isfinite(norm)
        scale = scale * torch.clamp(s["clip"] / (norm + 1e-6), max=1.0)
    g = g * scale.float()
    bits8 = s["bits"] == 8
    m0 = decode_m(f["m"], f["m_scale"]) if bits8 else f["m"]
    v0 = decode_v(f["v"], f["v_scale"]) if bits8 else f["v"]
    m = m0 * a + g * (1.0 - a)
    v = v0 * b + (g * (1.0 - b)) * g
    c1 = 1.0 - torch.pow(torch.full((), a, dtype=torch.float64, device=g.device), t)
    c2 = 1.0 - torch.pow(torch.full((), b, dtype=torch.float64, device=g.device), t)
    p = f["masters"] if s["master"] else f["params"].float()
    keep = (1.0 - lr * torch.tensor(s["decays"], dtype=torch.float64)).float().to(g.device).repeat_interleave(s["lengths"])
    q = p * keep - (m / (v.sqrt() * (1.0 / c2.sqrt()).float() + eps)) * (lr / c1).float()
    q = torch.where(fine, q, p)
    random = None
    if bits8 or (s["param"] == "bf16" and not s["master"]):
        key = (s["seed"] & MASK32) + ((t & MASK32) * 0x9E3779B9 & MASK32) & MASK32
        key = mix(mix(key) ^ ((s["seed"] >> 32 & MASK32) + s["index"] * 0x9E3779B9 & MASK32))
        place = torch.arange(g.numel(), device=g.device) - s["starts"].repeat_interleave(s["lengths"])
        random = mix(place ^ key.repeat_interleave(s["lengths"]))
    if bits8:
        code, e = encode_m(m, random)
        f["m"].view(torch.uint8).copy_(torch.where(fine, code.view(torch.uint8), f["m"].view(torch.uint8)))
        f["m_scale"].copy_(torch.where(fine, e, f["m_scale"]))
        code, e = encode_v(v, random)
        f["v"].copy_(torch.where(fine, code, f["v"]))
        f["v_scale"].copy_(torch.where(fine, e, f["v_scale"]))
    else:
        f["m"].copy_(torch.where(fine, m, m0))
        f["v"].copy_(torch.where(fine, v, v0))
    if s["master"]:
        f["masters"].copy_(q)
    if random is not None and not s["master"] and s["param"] == "bf16":
        r = (mix(random ^ 0x9E3779B9) & 0xFFFF).to(torch.int32)
        rounded = ((q.view(torch.int32) + r) >> 16 << 16).view(torch.float32)
        q = torch.where(fine & torch.isfinite(q), rounded, q)
    f["params"].copy_(q)
    s["control"][0] += fine.long()
    s["control"][1] += (~fine).long()


def answer_adamw(s):
    f = dict(s["flat"])
    del f["grads"]
    if s["bits"] == 8:  # the values that the codes stand for
        f["m"], f["v"] = decode_m(f["m"], f.pop("m_scale")), decode_v(f["v"], f.pop("v_scale"))
    f["counts"] = s["control"][:2]
    return f


# ---------------------------------------------------------------- one pass

def run(s):
    if not own:
        if s["op"] in ("ffn", "ffn_train"):
            return plain_ffn(s)
        if s["op"] == "residual":
            return plain_residual(s)
        plain_adamw(s)
        return answer_adamw(s)
    from paper_2312_08728_b200 import operators as ops
    if s["op"] == "ffn":
        return {"y": ops.gated_ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"], ACTIVATIONS.index(s["act"]))}
    if s["op"] == "ffn_train":
        weights, act = (s["w_gate"], s["w_up"], s["w_down"]), ACTIVATIONS.index(s["act"])
        y, saved = ops.gated_ffn(s["x"], *weights, act, save=True)
        dx, dw_gate, dw_up, dw_down = ops.gated_ffn_backward(s["dy"], s["x"], *weights, saved, act)
        return {"y": y, "dx": dx, "dw_gate": dw_gate, "dw_up": dw_up, "dw_down": dw_down}
    if s["op"] == "residual":
        residual, loss = ops.softmax_residual(s["logits"], s["y"])
        return {"residual": residual, "loss": loss}
    k = s["lists"]
    ops.adamw_step(k["params"], k["grads"], k["m"], k["v"], s["control"], weight_decay=s["decays"], max_norm=s["clip"],
                   grad_scale=s["gscale"], m_scale=k.get("m_scale"), v_scale=k.get("v_scale"), masters=k.get("masters"),
                   seed=s["seed"], **HYPER)
    return answer_adamw(s)


def work(case):
    if case["op"] in ("ffn", "ffn_train"):
        n, d, f, c = case["rows"], case["inputs"], case["hidden"], case["outputs"]
        values, flops = n * d + 2 * d * f + f * c + n * c, 2.0 * n * f * (2 * d + c)
        if case["op"] == "ffn_train":
            values, flops = 2 * values + n * c, 3.0 * flops   # dy is read; dx and the weights' gradients are written
        return {"bytes": 2.0 * values, "flops": flops}
    if case["op"] == "residual":
        n, c = case["rows"], case["classes"]
        return {"bytes": n * (2.0 * c * BYTES[case["type"]] + 8.0), "flops": 6.0 * n * c}
    total = sum(sizes_of(case))
    each = 2 * BYTES[case["param"]] + BYTES[case["grad"]] + (8 if case["master"] else 0) + (16 if case["bits"] == 32 else 4 + 4 / BLOCK)
    return {"bytes": float(total * each), "flops": 16.0 * total}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_ffn(s):
    x, wg, wu, wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
    gate, up = torch.mm(x, wg), torch.mm(x, wu)
    if s["act"] == "silu":
        value, slope = gate * torch.special.expit(gate), None
        slope = torch.special.expit(gate) + value * torch.special.expit(-gate)
    elif s["act"] == "sigmoid":
        value = torch.special.expit(gate)
        slope = value * torch.special.expit(-gate)
    elif s["act"] == "relu":
        value, slope = gate.clamp(min=0.0), (gate > 0).double()
    else:
        value = gate * torch.special.ndtr(gate)
        slope = torch.special.ndtr(gate) + gate * torch.exp(-gate.square() / 2) / math.sqrt(2 * math.pi)
    out = {"y": torch.mm(value * up, wd)}
    if s["op"] == "ffn_train":
        dy = s["dy"].double()
        back = torch.mm(dy, wd.t())
        out["dw_down"] = torch.mm((value * up).t(), dy)
        to_up = back * value
        out["dw_up"] = torch.mm(x.t(), to_up)
        to_gate = back * up * slope
        out["dw_gate"] = torch.mm(x.t(), to_gate)
        out["dx"] = torch.mm(to_gate, wg.t()) + torch.mm(to_up, wu.t())
    return out


def _exact_residual(s):
    # in slabs of rows: 64-bit copies of all logits at once would be large
    rows, classes = s["logits"].shape
    slab = max(1, 50_000_000 // classes)
    residual, loss = [], []
    for at in range(0, rows, slab):
        z, y = s["logits"][at:at + slab].double(), s["y"][at:at + slab].long()
        lse = torch.logsumexp(z, dim=1)
        one = torch.nn.functional.one_hot(y.clamp(min=0), classes).double() if classes * z.shape[0] < 2e7 else None
        r = torch.exp(z - lse[:, None])
        if one is not None:
            r = r - one
        else:
            r[torch.arange(len(y), device=y.device), y.clamp(min=0)] -= 1.0
        take = (y >= 0).double()
        residual.append(r * (take / rows)[:, None])
        loss.append((lse - z[torch.arange(len(y), device=y.device), y.clamp(min=0)]) * take)
    return {"residual": torch.cat(residual), "loss": torch.cat(loss)}


def _exact_adamw(s):
    f, t = s["flat"], int(s["control"][0]) + 1
    lr, beta1, beta2, eps = HYPER["lr"], HYPER["a"], HYPER["b"], HYPER["eps"]
    g = f["grads"].double() * s["gscale"]
    if s["clip"] > 0:
        g = g * min(1.0, s["clip"] / (float(torch.linalg.vector_norm(g)) + 1e-6))
    if s["bits"] == 8:
        code = f["m"].view(torch.uint8).long()
        exponent, fraction = (code >> 3) & 15, (code & 7).double() / 8
        size = torch.where(exponent > 0, (1 + fraction) * 2.0 ** (exponent - 7).double(), fraction * 2.0 ** -6)
        m = torch.where(code >= 128, -size, size) * 2.0 ** (f["m_scale"].double() - 134).repeat_interleave(BLOCK)
        code = f["v"].long()
        v = (1 + (code & 7).double() / 8) * 2.0 ** ((code >> 3).double() - 157 + f["v_scale"].double().repeat_interleave(BLOCK)) * (code > 0)
    else:
        m, v = f["m"].double(), f["v"].double()
    m += (1 - beta1) * (g - m)
    v += (1 - beta2) * (g * g - v)
    p = (f["masters"] if s["master"] else f["params"]).double()
    for tensor, (start, decay) in enumerate(zip(s["starts"].tolist(), s["decays"])):
        p[start:start + int(s["lengths"][tensor])] *= 1 - lr * decay
    p -= lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps)
    # moments in 8 bits are rounded up or down at random: next to a border either neighbour is right, so no one value is
    out = {"params": p, "m": m if s["bits"] == 32 else None, "v": v if s["bits"] == 32 else None, "counts": np.array([t, 0])}
    if s["master"]:
        out["masters"] = p
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("ffn", "ffn_train"):
        return _exact_ffn(s)
    return _exact_residual(s) if case["op"] == "residual" else _exact_adamw(s)
