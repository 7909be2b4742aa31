"""Cases for the operators around the gated block: the norm with the residual's addition (for scoring, for training, with
8-bit output), rows quantised behind the gate, the product in 8-bit integers, log probabilities with entropy and top
alternatives (alone, and with their gradient), and dropout.

Each case has an entry "op": "norm", "gate", "int8", "logprobs" or "dropout".  `run` computes the operator with elementary
torch operations where `own` is false, and calls the library where it is true.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
ACTIVATIONS = ("silu", "gelu", "relu", "sigmoid")   # in the library's numbering: 0, 1, 2, 3
EPS = 1e-6
LEAST = 2.0 ** -120                                 # rows that nowhere exceed this are zeros in 8 bits
MASK32 = 0xFFFFFFFF


def listed():
    return [
        # ---- norm of a row plus its residual
        # one row on its way to an 8-bit product: a request that is answered as it comes
        dict(name="norm one row int8", op="norm", mode="int8", rows=1, width=4096, type="bf16", weight="fp32", residual=True, extra=0),
        # a mini-batch of an odd width, rows that are a slice of a wider buffer, forward and backward
        dict(name="norm odd width train", op="norm", mode="train", rows=777, width=501, type="fp16", weight="same", residual=False, extra=12),
        # a large mini-batch of a wide residual stream, forward and backward
        dict(name="norm large train", op="norm", mode="train", rows=8192, width=4096, type="bf16", weight="fp32", residual=True, extra=0),
        # ---- the hidden layer of the gated block between two 8-bit products: gate and value stand side by side in one matrix
        dict(name="gate one row", op="gate", rows=1, width=11008, type="bf16", act="silu"),
        dict(name="gate many rows", op="gate", rows=4096, width=11008, type="bf16", act="silu"),
        # ---- product in 8-bit integers: tokens x inputs -> outputs
        # one token
        dict(name="int8 one token", op="int8", rows=1, inputs=4096, outputs=11008, type="bf16", bias=False, extra=0),
        # a handful of tokens, odd sizes, a bias, rows that no copy engine reads
        dict(name="int8 few odd", op="int8", rows=29, inputs=1371, outputs=2501, type="fp16", bias=True, extra=7),
        # a buffer's rows scored in one call
        dict(name="int8 many tokens", op="int8", rows=4096, inputs=4096, outputs=11008, type="bf16", bias=False, extra=0),
        # ---- log probabilities
        # the answer of one request over many classes, with its five best alternatives, some classes ruled out
        dict(name="logprobs one row", op="logprobs", train=False, rows=1, classes=50257, type="bf16", top=5, skipped=0, ruled_out=0.3),
        # a large batch scored with 20 alternatives, and the gradient of log probabilities and entropies
        dict(name="logprobs many train", op="logprobs", train=True, rows=8191, classes=50257, type="bf16", top=20, skipped=40, ruled_out=0.0),
        # ---- dropout
        # the mini-batch of a small model, added to the residual stream
        dict(name="dropout small", op="dropout", rows=777, width=501, type="fp16", rate=0.1, residual=True, extra=0),
        # a large hidden layer
        dict(name="dropout large", op="dropout", rows=16384, width=11008, type="bf16", rate=0.25, residual=False, extra=0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _eights(rng, n):
    return -(-n // 8) * 8 if rng.random() < 0.6 else n   # most models have widths of a multiple of eight


def draw(rng):
    op = rng.choice(["norm", "norm", "gate", "int8", "int8", "logprobs", "logprobs", "dropout"])
    if op == "norm":
        width = _eights(rng, _log(rng, 2, 20_000))
        return dict(op=op, mode=rng.choice(["plain", "train", "int8"]), rows=_log(rng, 1, min(16_384, 32_000_000 // width)), width=width,
                    type=rng.choice(["bf16", "fp16", "fp32"]), weight=rng.choice(["same", "fp32"]), residual=rng.random() < 0.5,
                    extra=rng.choice([0, 0, 1, 8]))
    if op == "gate":
        width = _eights(rng, _log(rng, 2, 16_384))
        return dict(op=op, rows=_log(rng, 1, min(16_384, 40_000_000 // width)), width=width, type=rng.choice(["bf16", "fp16", "fp32"]),
                    act=rng.choice(ACTIVATIONS))
    if op == "int8":
        return dict(op=op, rows=_log(rng, 1, 4096), inputs=_eights(rng, _log(rng, 16, 4096)), outputs=_eights(rng, _log(rng, 2, 8192)),
                    type=rng.choice(["bf16", "fp16", "fp32"]), bias=rng.random() < 0.5, extra=rng.choice([0, 0, 1, 16]))
    if op == "logprobs":
        classes = _log(rng, 2, 130_000)
        rows = _log(rng, 1, min(16_384, 200_000_000 // classes))
        return dict(op=op, train=rng.random() < 0.5, rows=rows, classes=classes, type=rng.choice(["bf16", "fp16", "fp32"]),
                    top=min(classes, rng.choice([0, 1, 5, 20, 32])), skipped=rng.choice([0, rows // 5]), ruled_out=rng.choice([0.0, 0.0, 0.5]))
    width = _eights(rng, _log(rng, 2, 16_384))
    return dict(op=op, rows=_log(rng, 1, min(65_536, 100_000_000 // width)), width=width, type=rng.choice(["bf16", "fp16", "fp32"]),
                rate=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5, extra=rng.choice([0, 0, 1, 8]))


# ---------------------------------------------------------------- inputs

def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _rows(gen, n, width, extra, dtype, scale=1.0):
    """[n, width], rows of a wider buffer where extra > 0."""
    return _normal(gen, (n, width + extra), dtype, scale)[:, :width]


def _bytes(gen, n, width, extra):
    """Rows in 8 bits as they come out of the quantisation of normal values: the largest of a row at 127."""
    v = torch.randn((n, width + extra), generator=gen, device="cuda", dtype=torch.float32)
    return (v * (127.0 / v.abs().amax(dim=1, keepdim=True))).round().to(torch.int8)[:, :width]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s, t = dict(case), TYPES[case["type"]]
    if case["op"] == "norm":
        n, d, extra = case["rows"], case["width"], case["extra"]
        s["x"] = _rows(gen, n, d, extra, t)
        # a residual stream: a few columns are much larger than the others
        spread = torch.exp2(torch.randint(0, 12, (d,), generator=gen, device="cuda").float().sub_(7).clamp_(min=0))
        s["r"] = (_rows(gen, n, d, extra, torch.float32) * spread).to(t) if case["residual"] else None
        s["w"] = (1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(t if case["weight"] == "same" else torch.float32)
        if case["mode"] == "train":
            s["dy"] = _normal(gen, (n, d), t, 0.1)
            s["dtotal"] = _normal(gen, (n, d), t, 0.1) if case["residual"] else None
    elif case["op"] == "gate":
        s["both"] = _normal(gen, (case["rows"], 2 * case["width"]), t)
    elif case["op"] == "int8":
        n, d, c = case["rows"], case["inputs"], case["outputs"]
        s["q"], s["w"] = _bytes(gen, n, d, case["extra"]), _bytes(gen, c, d, case["extra"])
        s["q_scale"] = torch.rand(n, generator=gen, device="cuda") * 0.03 + 0.01
        s["w_scale"] = (torch.rand(c, generator=gen, device="cuda") * 0.03 + 0.01) * d ** -0.5
        s["bias"] = _normal(gen, (c,), torch.float32) if case["bias"] else None
    elif case["op"] == "logprobs":
        n, c = case["rows"], case["classes"]
        z = torch.randn((n, c), generator=gen, device="cuda", dtype=torch.float32).mul_(3.0)
        s["y"] = torch.randint(0, c, (n,), generator=gen, device="cuda", dtype=torch.int32)
        if case["ruled_out"]:   # never the label's class
            out = torch.rand((n, c), generator=gen, device="cuda") < case["ruled_out"]
            out.scatter_(1, s["y"].long().unsqueeze(1), False)
            z.masked_fill_(out, -math.inf)
        s["logits"] = z.to(t)
        s["y"][:case["skipped"]] = -1
        if case["train"]:       # an advantage per row, and the weight of the entropy
            s["dlogprob"] = torch.randn(n, generator=gen, device="cuda") / n
            s["dentropy"] = torch.rand(n, generator=gen, device="cuda") * 0.1 / n
    else:
        n, d, extra = case["rows"], case["width"], case["extra"]
        s["x"] = _rows(gen, n, d, extra, t)
        s["r"] = _rows(gen, n, d, extra, t) if case["residual"] else None
        s["seed"] = int(seed) * 7919 + 5
        s["step"] = torch.full((1,), int(seed) % 1000, dtype=torch.int64, device="cuda")   # as the updates are counted
    return s


# ---------------------------------------------------------------- plain forms

def quantized(y, dtype):
    """Rows in 8 bits: the values that they stand for, and the scale of each row."""
    top = y.abs().amax(dim=1, keepdim=True)
    some = top >= LEAST
    q = torch.where(some, (y * (127.0 / torch.where(some, top, torch.ones_like(top)))).round(), torch.zeros_like(y))
    scale = torch.where(some, top / 127.0, torch.zeros_like(top))
    return (q * scale).to(dtype), scale.squeeze(1)


def plain_norm(s):
    t = s["x"].dtype
    total = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(t)   # the norm is that of the stored sum
    v, w = total.float(), s["w"].float()
    rstd = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    y = v * rstd * w
    out = {} if s["r"] is None else {"total": total}
    if s["mode"] == "int8":
        out["values"], out["scale"] = quantized(y, t)
        return out
    out["y"] = y.to(t)
    if s["mode"] == "train":
        dy = s["dy"].float()
        g, unit = dy * w, v * rstd
        dx = rstd * (g - unit * (g * unit).mean(dim=1, keepdim=True))
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        out["dx"], out["dw"] = dx.to(t), (dy * unit).sum(dim=0).to(s["w"].dtype)
    return out


def plain_gate(s):
    g, u = s["both"][:, :s["width"]].float(), s["both"][:, s["width"]:].float()
    if s["act"] == "relu":
        h = g * (g > 0)
    elif s["act"] == "gelu":
        h = g * (0.5 * (1.0 + torch.erf(g * math.sqrt(0.5))))
    else:
        h = 1.0 / (1.0 + torch.exp(-g))
        h = g * h if s["act"] == "silu" else h
    values, scale = quantized(h * u, s["both"].dtype)
    return {"values": values, "scale": scale}


def plain_int8(s):
    sums = s["q"].double() @ s["w"].double().T      # whole numbers up to 2^31: 32-bit floats would lose some
    y = sums.float() * s["q_scale"].unsqueeze(1) * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(TYPES[s["type"]])}


def plain_logprobs(s):
    z, y, k = s["logits"].float(), s["y"].long(), s["top"]
    n, c = z.shape
    with_label = (y >= 0) & (y < c)
    top = z.amax(dim=1, keepdim=True)
    below = z - top
    p = torch.exp(below)
    total = p.sum(dim=1, keepdim=True)
    p = p / total
    lse = torch.log(total) + top
    logp = z - lse
    finite = torch.where(p > 0, logp, torch.zeros_like(logp))        # ruled-out classes have no part in the entropy
    entropy = -(p * finite).sum(dim=1, keepdim=True)
    at = y.clamp(0, c - 1).unsqueeze(1)
    picked = logp.gather(1, at).squeeze(1)
    out = {"logprob": torch.where(with_label, picked, torch.zeros_like(picked)), "entropy": entropy.squeeze(1)}
    if k > 0:   # ties go to the lowest index: order by the value's bits, then by the place
        bits = (z + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32 + (c - 1 - torch.arange(c, device=z.device))
        index = order.topk(k, dim=1).indices
        out["index"], out["alternatives"] = index.to(torch.int32), logp.gather(1, index)
    if s["train"]:
        dl = torch.where(with_label, s["dlogprob"], torch.zeros_like(s["dlogprob"])).unsqueeze(1)
        dz = -p * (dl + s["dentropy"].unsqueeze(1) * (finite + entropy))
        dz.scatter_add_(1, at, dl)
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def philox(counter, key):
    """Philox4x32-10 (Salmon et al. 2011) on int64 tensors that hold 32-bit words."""
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57       # (64-bit products wrap; their upper halves are taken as unsigned)
        c0, c1, c2, c3 = ((b >> 32) & MASK32) ^ c1 ^ k0, b & MASK32, ((a >> 32) & MASK32) ^ c3 ^ k1, a & MASK32
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    return c0, c1, c2, c3


def kept(s):
    """Which values stay: 16 bits for each, eight values to a block of the generator, in the order of the rows."""
    n, d = s["rows"], s["width"]
    block = torch.arange(-(-n * d // 8), device="cuda")
    zero = torch.zeros_like(block)
    words = philox((block & MASK32, block >> 32, zero + (s["step"][0] & MASK32), zero + 0x44524F50),
                   (s["seed"] & MASK32, s["seed"] >> 32 & MASK32))
    halves = torch.stack([half for w in words for half in (w & 0xFFFF, w >> 16)], dim=1).view(-1)
    return (halves[:n * d] >= round(s["rate"] * 65536)).view(n, d)


def plain_dropout(s):
    out_of = round(s["rate"] * 65536)
    y = torch.where(kept(s), s["x"].float() * (65536.0 / (65536 - out_of)), torch.zeros((), device="cuda"))
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(s["x"].dtype)}


# ---------------------------------------------------------------- one pass

def _values(q, scale, dtype):
    """What rows in 8 bits stand for."""
    out = torch.empty(q.shape, dtype=dtype, device=q.device)
    return torch.mul(q, scale.unsqueeze(1), out=out)


def run(s):
    if not own:
        return {"norm": plain_norm, "gate": plain_gate, "int8": plain_int8, "logprobs": plain_logprobs, "dropout": plain_dropout}[s["op"]](s)
    from paper_2312_08728_b200 import operators as ops
    if s["op"] == "norm":
        if s["mode"] == "int8":
            q, scale, total = ops.rms_norm_int8(s["x"], s["w"], residual=s["r"], eps=EPS)
            out = {"values": _values(q, scale, s["x"].dtype), "scale": scale}
        elif s["mode"] == "train":
            y, total, rstd = ops.rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS, save=True)
            dx, dw = ops.rms_norm_backward(s["dy"], total, s["w"], rstd, dtotal=s["dtotal"])
            out = {"y": y, "dx": dx, "dw": dw}
        else:
            y, total = ops.rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS)
            out = {"y": y}
        return out if s["r"] is None else {"total": total, **out}
    if s["op"] == "gate":
        q, scale = ops.quantize_rows(s["both"][:, s["width"]:], gate=s["both"][:, :s["width"]], activation=ACTIVATIONS.index(s["act"]))
        return {"values": _values(q, scale, s["both"].dtype), "scale": scale}
    if s["op"] == "int8":
        return {"y": ops.int8_linear(s["q"], s["q_scale"], s["w"], s["w_scale"], bias=s["bias"], dtype=TYPES[s["type"]])}
    if s["op"] == "logprobs":
        logprob, entropy, index, alternatives, *saved = ops.log_probs(s["logits"], s["y"], top=s["top"], save=s["train"])
        out = {"logprob": logprob, "entropy": entropy}
        if s["top"] > 0:
            out["index"], out["alternatives"] = index, alternatives
        if s["train"]:
            out["dlogits"] = ops.log_probs_backward(s["dlogprob"], s["dentropy"], s["logits"], s["y"], *saved)
        return out
    return {"y": ops.dropout(s["x"], s["rate"], s["seed"], step=s["step"], residual=s["r"])}


def work(case):
    e = BYTES[case["type"]]
    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        ins = 2 if case["residual"] else 1
        size = n * d * (ins * e + (e if case["residual"] else 0) + (1 if case["mode"] == "int8" else e))
        w = d * (e if case["weight"] == "same" else 4)
        if case["mode"] == "train":     # dy and the sum's gradient come beside what the forward pass reads, dx and dw are written
            size += n * d * e * (3 if case["residual"] else 2)
            w *= 2
        return {"bytes": float(size + w), "flops": n * d * (16.0 if case["mode"] == "train" else 5.0)}
    if case["op"] == "gate":
        return {"bytes": case["rows"] * (case["width"] * (2.0 * e + 1.0) + 4.0), "flops": 8.0 * case["rows"] * case["width"]}
    if case["op"] == "int8":
        n, d, c = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": n * d + d * c + n * c * e + 4.0 * (n + c), "flops": 2.0 * n * d * c}
    if case["op"] == "logprobs":
        n, c = case["rows"], case["classes"]
        return {"bytes": n * (c * e * (2.0 if case["train"] else 1.0) + 12.0 + 8.0 * case["top"]), "flops": n * c * (12.0 if case["train"] else 6.0)}
    n, d = case["rows"], case["width"]
    return {"bytes": float(n * d * e * (3 if case["residual"] else 2)), "flops": 12.0 * n * d}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_quantized(y):
    step = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / 127
    codes = torch.where(step[:, None] * 127 < LEAST, torch.zeros_like(y), torch.round(y / step[:, None]))
    step = torch.where(step * 127 < LEAST, torch.zeros_like(step), step)
    return codes * step[:, None], step


def _exact_norm(s):
    total = s["x"].double()
    out = {}
    if s["r"] is not None:
        total = (total + s["r"].double()).to(s["x"].dtype).double()
        out["total"] = total
    total = total.clone().requires_grad_(True)
    w = s["w"].double().requires_grad_(True)
    with torch.enable_grad():
        y = w * total / torch.sqrt(total.square().sum(dim=1, keepdim=True) / total.shape[1] + EPS)
    if s["mode"] == "int8":
        out["values"], out["scale"] = _exact_quantized(y.detach())
        return out
    out["y"] = y.detach()
    if s["mode"] == "train":
        dx, dw = torch.autograd.grad(y, (total, w), s["dy"].double())
        out["dx"], out["dw"] = dx if s["dtotal"] is None else dx + s["dtotal"].double(), dw
    return out


def _exact_gate(s):
    g, u = s["both"].double().chunk(2, dim=1)
    h = {"silu": lambda: g * torch.special.expit(g), "gelu": lambda: g * torch.special.ndtr(g), "relu": lambda: g.clamp(min=0),
         "sigmoid": lambda: torch.special.expit(g)}[s["act"]]()
    values, scale = _exact_quantized(h * u)
    return {"values": values, "scale": scale}


def _exact_int8(s):
    x, w = s["q"].double() * s["q_scale"].double()[:, None], s["w"].double() * s["w_scale"].double()[:, None]
    y = torch.einsum("nk,ck->nc", x, w)
    return {"y": y if s["bias"] is None else y + s["bias"].double()}


def _exact_logprobs(s):
    # in slabs of rows: 64-bit copies of all logits at once would be large
    rows, classes = s["logits"].shape
    slab = max(1, 50_000_000 // classes)
    parts = []
    for at in range(0, rows, slab):
        z = s["logits"][at:at + slab].double().requires_grad_(s["train"])
        y = s["y"][at:at + slab].long()
        here = torch.arange(len(y), device=y.device)
        with torch.enable_grad():
            logp = z - torch.logsumexp(z, dim=1, keepdim=True)
            some = torch.where(torch.isinf(z), torch.zeros_like(z), logp)       # 0 log 0 = 0
            entropy = -(torch.exp(logp) * some).sum(dim=1)
            logprob = torch.where(y >= 0, some[here, y.clamp(min=0)], torch.zeros_like(entropy))
        part = {"logprob": logprob.detach(), "entropy": entropy.detach()}
        if s["top"] > 0:
            best = torch.sort(z.detach(), dim=1, descending=True, stable=True).indices[:, :s["top"]]
            part["index"], part["alternatives"] = best.to(torch.int32), logp.detach().gather(1, best)
        if s["train"]:
            (part["dlogits"],) = torch.autograd.grad((logprob, entropy), z, (s["dlogprob"][at:at + slab].double(), s["dentropy"][at:at + slab].double()))
        parts.append(part)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_dropout(s):
    share = 1.0 - round(s["rate"] * 65536) / 65536
    y = s["x"].double() / share * kept(s)       # (which values stay is a matter of whole numbers)
    return {"y": y if s["r"] is None else y + s["r"].double()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "gate": _exact_gate, "int8": _exact_int8, "logprobs": _exact_logprobs, "dropout": _exact_dropout}[case["op"]](s)
