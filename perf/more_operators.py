"""What a served model needs around its quantized attention, and what measures it, as cases that can be timed: the norm with
the residual's addition and an 8-bit output, the 8-bit product with activation, gate and residual in its epilogue, the log
probabilities of given tokens with entropy and alternatives, and the distillation loss on a teacher's top logits with its gradient.

Every operator has its plain form here (elementary torch operations in 32 bits, rounded once at the end) and, with `own` set, the
calls that a user makes of this package.  Sizes: the 7B-, 72B- and 2B-class layers of the package's workloads (hidden 3584 / 8192 /
1536, inner width 18944 / 29568 / 8960), and vocabularies of 32,000 to 131,072 entries, odd ones among them.
"""
import math

import torch

own = False

FLOOR = 1e-5        # smallest |.| maximum that a quantization step is made from
EPS = 1e-6


def listed():
    return [
        # one token of a chat between two layers: launch latency
        {"name": "norm: 1 token, 3584", "op": "norm", "tokens": 1, "width": 3584, "residual": True, "scales": True, "codes": True, "pitch": 0},
        # the norm before the vocabulary's product, kept in 16 bits, for a short prompt of odd length out of a wider buffer
        {"name": "norm: 67 tokens, 1536, 16 bits", "op": "norm", "tokens": 67, "width": 1536, "residual": False, "scales": False, "codes": False,
         "pitch": 64},
        # a long prompt of the 72B-class layer: bytes
        {"name": "norm: 8192 tokens, 8192", "op": "norm", "tokens": 8192, "width": 8192, "residual": True, "scales": True, "codes": True, "pitch": 0},
        # one token through the 7B-class gate and up projections, in one product: the weights' bytes
        {"name": "product: 1 token, gated", "op": "product", "tokens": 1, "c_in": 3584, "c_out": 37888, "act": "silu", "gated": True,
         "bias": False, "residual": False},
        # a short prompt through the 2B-class down projection, added to the residual stream
        {"name": "product: 201 tokens, residual", "op": "product", "tokens": 201, "c_in": 8960, "c_out": 1536, "act": "none", "gated": False,
         "bias": False, "residual": True},
        # patches of an image through a vision layer: bias and GELU, odd number of rows
        {"name": "product: 1025 patches, GELU", "op": "product", "tokens": 1025, "c_in": 1280, "c_out": 5120, "act": "gelu", "gated": False,
         "bias": True, "residual": False},
        # a long prompt, or a calibration batch, through the 7B-class gate and up projections: the tensor cores
        {"name": "product: 8192 tokens, gated", "op": "product", "tokens": 8192, "c_in": 3584, "c_out": 37888, "act": "silu", "gated": True,
         "bias": False, "residual": False},
        # the answer of one chat: one row over many SMs, with its alternatives
        {"name": "logprobs: 1 answer, top 20", "op": "logprobs", "tokens": 1, "vocab": 131072, "top": 20, "entropy": True, "bits": 16, "scale": 1.0},
        # answers of a batch in 32 bits at a temperature, odd vocabulary
        {"name": "logprobs: 64 answers, 32 bits", "op": "logprobs", "tokens": 64, "vocab": 50001, "top": 5, "entropy": True, "bits": 32, "scale": 1.25},
        # a calibration batch through the full-precision model: its alternatives become the teacher's logits
        {"name": "logprobs: 4096 tokens, top 64", "op": "logprobs", "tokens": 4096, "vocab": 131072, "top": 64, "entropy": True, "bits": 16, "scale": 1.0},
        # the loss alone, over an odd vocabulary
        {"name": "distill: 511 tokens, loss", "op": "distill", "tokens": 511, "vocab": 65537, "top": 20, "bits": 16, "grad": False, "scale": 0.5},
        # a calibration batch through the quantized model: loss and gradient
        {"name": "distill: 4096 tokens, gradient", "op": "distill", "tokens": 4096, "vocab": 131072, "top": 64, "bits": 16, "grad": True, "scale": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("norm", "product", "product", "logprobs", "logprobs", "distill", "distill"))
    if op == "norm":
        width = 16 * _log(rng, 8, 1848)
        codes = rng.random() < 0.75
        return {"op": op, "tokens": _log(rng, 1, min(16384, 8192 * 8192 // width)), "width": width, "residual": rng.random() < 0.7,
                "scales": codes and rng.random() < 0.7, "codes": codes, "pitch": rng.choice((0, 0, 8, 1000))}
    if op == "product":
        act = rng.choice(("none", "silu", "silu", "gelu", "gelu_tanh"))
        gated = act != "none" and rng.random() < 0.6
        c_in, c_out = 16 * _log(rng, 8, 1184), _log(rng, 200, 18944)
        most = 8192 * 3584 * 18944 // (c_in * c_out)
        return {"op": op, "tokens": _log(rng, 1, min(8192, most)), "c_in": c_in, "c_out": 2 * c_out if gated else c_out, "act": act, "gated": gated,
                "bias": rng.random() < 0.5, "residual": act == "none" or rng.random() < 0.3}
    bits = rng.choice((16, 16, 32))
    vocab = _log(rng, 1000, 131072)
    case = {"op": op, "tokens": _log(rng, 1, min(4096, 4096 * 131072 * 16 // (bits * vocab))), "vocab": vocab, "bits": bits,
            "scale": rng.choice((1.0, 1.0, 0.5, 1.25))}
    if op == "logprobs":
        return {**case, "top": rng.choice((0, 1, 5, 20, 64, 128)), "entropy": rng.random() < 0.6}
    return {**case, "top": rng.choice((1, 8, 20, 64, 128)), "grad": rng.random() < 0.7}


def _width(case):
    return case["c_out"] // 2 if case["gated"] else case["c_out"]


def work(case):
    n = case["tokens"]
    if case["op"] == "norm":
        c = case["width"]
        moved = 2 * n * c + (4 * n * c if case["residual"] else 0)      # x in; the residual in, the sum out
        moved += 3 * n * c + 4 * n if case["codes"] else 2 * n * c      # codes, the values they stand for, steps; or 16 bits
        return {"bytes": moved + 2 * c * (2 if case["scales"] else 1), "flops": 8 * n * c}
    if case["op"] == "product":
        ci, co, w = case["c_in"], case["c_out"], _width(case)
        moved = n * ci + ci * co + 4 * (n + co) + (2 * co if case["bias"] else 0) + (2 * n * w if case["residual"] else 0) + 2 * n * w
        return {"bytes": moved, "flops": 2 * n * ci * co}
    v, size, k = case["vocab"], case["bits"] // 8, case["top"]
    if case["op"] == "logprobs":
        return {"bytes": n * (v * size + 4 + 4 + (4 if case["entropy"] else 0) + 8 * k), "flops": (6 if case["entropy"] else 4) * n * v}
    return {"bytes": n * (v * size * (2 if case["grad"] else 1) + 8 * k + 8), "flops": (7 if case["grad"] else 4) * n * v}


# ------------------------------------------------------------------------------------------------ inputs

def _codes(x):
    """int8 codes and steps of the rows of x."""
    step = x.abs().amax(1, keepdim=True).clamp_min(FLOOR) / 127
    return torch.round(x / step).to(torch.int8), step.flatten().contiguous()


def _norm_inputs(case, g, dev):
    n, c = case["tokens"], case["width"]

    def stream():
        x = torch.randn(n, c + case["pitch"], generator=g, device=dev)
        x[:, torch.randint(0, c, (4,), generator=g, device=dev)] *= 8       # activations keep a few large channels
        return x.bfloat16()[:, :c]
    s = {"x": stream(), "residual": stream() if case["residual"] else None,
         "w": (1 + 0.2 * torch.randn(c, generator=g, device=dev)).bfloat16(), "s": None, "codes": case["codes"]}
    if case["scales"]:
        s["s"] = torch.exp(0.5 * torch.randn(c, generator=g, device=dev)).bfloat16()
    return s


def _product_inputs(case, g, dev):
    n, ci, co = case["tokens"], case["c_in"], case["c_out"]
    x = torch.randn(n, ci, generator=g, device=dev)
    x[:, torch.randint(0, ci, (4,), generator=g, device=dev)] *= 8
    xq, t = _codes(x)
    wq, u = _codes(torch.randn(co, ci, generator=g, device=dev) * (1.5 * ci ** -0.5))
    return {"xq": xq, "t": t, "wq": wq, "u": u, "act": case["act"], "gated": case["gated"],
            "bias": torch.randn(co, generator=g, device=dev).bfloat16() if case["bias"] else None,
            "residual": torch.randn(n, _width(case), generator=g, device=dev).bfloat16() if case["residual"] else None}


def _logits(case, g, dev):
    """Rows with a broad floor of unlikely tokens and some likely ones."""
    n, v = case["tokens"], case["vocab"]
    z = torch.randn(n, v, generator=g, device=dev).mul_(2)
    likely = (torch.randint(0, v, (n, 1), generator=g, device=dev) + torch.arange(24, device=dev) * (v // 24)) % v     # no token twice
    z.scatter_add_(1, likely, 4 + 9 * torch.rand(n, 24, generator=g, device=dev))
    return (z if case["bits"] == 32 else z.bfloat16()), likely


def _logprobs_inputs(case, g, dev):
    z, likely = _logits(case, g, dev)
    ids = likely[:, 0].to(torch.int32).contiguous()
    if case["tokens"] > 1:
        ids[torch.rand(case["tokens"], generator=g, device=dev) < 0.05] = -1    # rows of a padded batch
    return {"z": z, "ids": ids, "top": case["top"], "entropy": case["entropy"], "scale": case["scale"]}


def _distill_inputs(case, g, dev):
    z, _ = _logits(case, g, dev)
    teacher = torch.randn(z.shape, generator=g, device=dev).mul_(0.7).add_(z)
    top, ids = torch.topk(teacher, case["top"], dim=1)
    del teacher
    weights = torch.exp(torch.randn(case["tokens"], generator=g, device=dev))   # the importance of tokens
    if case["tokens"] > 1:
        weights[torch.rand(case["tokens"], generator=g, device=dev) < 0.1] = 0  # and those that do not count
    return {"z": z, "top": top.contiguous(), "ids": ids.to(torch.int32).contiguous(), "weights": weights / case["tokens"], "grad": case["grad"],
            "scale": case["scale"]}


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    s = {"norm": _norm_inputs, "product": _product_inputs, "logprobs": _logprobs_inputs, "distill": _distill_inputs}[case["op"]](case, g, dev)
    s["op"] = case["op"]
    if own:     # what a program makes once: the quantizer's settings, a workspace
        from paper_2602_07899_b200 import tlq
        s["tlq"] = tlq
        if case["op"] == "norm":
            s["cfg"] = tlq.config(tlq.W8A8_SYM)
        if case["op"] == "product":
            s["ws"] = tlq.linear_workspace(case["tokens"], case["c_in"], case["c_out"], dev)
            s["number"] = {"none": tlq.ACT_NONE, "silu": tlq.ACT_SILU, "gelu": tlq.ACT_GELU, "gelu_tanh": tlq.ACT_GELU_TANH}[case["act"]]
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_norm(s):
    out = {}
    h = s["x"]
    if s["residual"] is not None:
        h = out["h"] = (h.float() + s["residual"].float()).bfloat16()
    h = h.float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["w"].float()
    if not s["codes"]:
        return {**out, "y": y.bfloat16()}
    if s["s"] is not None:
        y = y * (1 / s["s"].float())
    step = y.abs().amax(1, keepdim=True).clamp_min(FLOOR) / 127
    return {**out, "values": (torch.round(y / step) * step).bfloat16(), "steps": step[:, 0]}


def _activated(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _plain_product(s):
    y = (s["xq"].float() @ s["wq"].float().t()) * s["t"][:, None] * s["u"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _activated(y[:, ::2], s["act"]) * y[:, 1::2] if s["gated"] else _activated(y, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.bfloat16()


def _softmax_parts(z, scale):
    """scale (z - its maximum), the sum of their exponentials, and the maximum."""
    top = z.amax(1, keepdim=True)
    d = (z - top) * scale
    return d, torch.exp(d).sum(1, keepdim=True), top


def _plain_logprobs(s):
    z = s["z"].float()
    d, total, top = _softmax_parts(z, s["scale"])
    log_total = total.log()
    ids = s["ids"].long()
    logp = (d.gather(1, ids.clamp_min(0)[:, None]) - log_total)[:, 0]
    out = {"logp": torch.where(ids < 0, torch.zeros_like(logp), logp), "lse": (top * s["scale"] + log_total)[:, 0]}
    if s["entropy"]:
        out["entropy"] = (log_total - (torch.exp(d) * d).sum(1, keepdim=True) / total)[:, 0]
    if s["top"]:
        bits = (z + 0.0).view(torch.int32)                  # in the order of the values, the lower index first among equals
        rank = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long().mul_(1 << 32)
        rank += (1 << 31) - torch.arange(z.shape[1], device=z.device)
        at = torch.topk(rank, s["top"], dim=1).indices
        out["top_ids"], out["top_logp"] = at.to(torch.int32), d.gather(1, at) - log_total
    return out


def _plain_distill(s):
    scale, w = s["scale"], s["weights"][:, None]
    d, total, _ = _softmax_parts(s["z"].float(), scale)
    t = (s["top"] - s["top"].amax(1, keepdim=True)) * scale
    lt = t - torch.exp(t).sum(1, keepdim=True).log()
    p, ids = torch.exp(lt), s["ids"].long()
    loss = w * (p * (lt - (d.gather(1, ids) - total.log()))).sum(1, keepdim=True)
    if not s["grad"]:
        return {"loss": loss[:, 0]}
    q = torch.exp(d) / total
    grad = q.scatter_add_(1, ids, -p) * (w * scale)
    return {"loss": loss[:, 0], "grad": grad.to(s["z"].dtype)}


def run(s):
    if not own:
        return {"norm": _plain_norm, "product": _plain_product, "logprobs": _plain_logprobs, "distill": _plain_distill}[s["op"]](s)
    t = s["tlq"]
    if s["op"] == "norm":
        r = t.tlq_norm_quantize(s["x"], s["w"], s["cfg"], residual=s["residual"], s=s["s"], eps=EPS, want_codes=s["codes"], want_values=s["codes"],
                                want_y=not s["codes"])
        return {k: r[k] for k in ("h", "y", "values", "steps") if r[k] is not None and (k != "h" or s["residual"] is not None)}
    if s["op"] == "product":
        return t.tlq_linear_i8_act(s["xq"], s["t"], s["wq"], s["u"], s["bias"], act=s["number"], gated=s["gated"], residual=s["residual"],
                                   workspace=s["ws"])
    if s["op"] == "logprobs":
        r = t.tlq_token_logprobs(s["z"], s["ids"], top_k=s["top"], scale=s["scale"], want_entropy=s["entropy"], want_lse=True)
        return {k: v for k, v in r.items() if v is not None}
    loss, grad = t.tlq_distill_loss(s["z"], s["ids"], s["top"], s["weights"], scale=s["scale"], want_grad=s["grad"])
    return {"loss": loss, "grad": grad} if s["grad"] else {"loss": loss}


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_norm(s):
    """Row by row in pieces, as the definition reads."""
    x, r = s["x"].double(), s["residual"]
    out = {}
    if r is not None:
        x = (x + r.double()).bfloat16().double()    # the residual stream is held in 16 bits
        out["h"] = x
    y = x / (x.square().sum(1, keepdim=True) / x.shape[1] + EPS).sqrt() * s["w"].double()
    if not s["codes"]:
        return {**out, "y": y}
    if s["s"] is not None:
        y = y / s["s"].double()
    step = y.abs().max(1, keepdim=True).values.clamp(min=FLOOR) / 127
    return {**out, "values": torch.round(y / step) * step, "steps": step.flatten()}


def _exact_product(s):
    y = torch.mm(s["xq"].double(), s["wq"].double().t()) * torch.outer(s["t"].double(), s["u"].double())
    if s["bias"] is not None:
        y += s["bias"].double()
    z = y[:, 0::2] if s["gated"] else y
    z = {"none": lambda v: v, "silu": lambda v: v * torch.sigmoid(v), "gelu": lambda v: v * torch.special.ndtr(v),
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[s["act"]](z)
    if s["gated"]:
        z = z * y[:, 1::2]
    return z if s["residual"] is None else z + s["residual"].double()


def _rows_at_once(v):
    return max(1, (1 << 26) // v)


def _exact_logprobs(s):
    z, k, got = s["z"], s["top"], []
    for part, ids in zip(z.split(_rows_at_once(z.shape[1])), s["ids"].split(_rows_at_once(z.shape[1]))):
        a = part.double() * s["scale"]
        lp = torch.log_softmax(a, 1)
        row = {"logp": torch.where(ids < 0, 0.0, lp[torch.arange(len(ids), device=z.device), ids.clamp(min=0).long()]), "lse": torch.logsumexp(a, 1)}
        if s["entropy"]:
            row["entropy"] = -(lp.exp() * lp).sum(1)
        if k:
            at = torch.sort(part.float(), dim=1, descending=True, stable=True).indices[:, :k]
            row["top_ids"], row["top_logp"] = at.to(torch.int32), lp.gather(1, at)
        got.append(row)
    return {name: torch.cat([r[name] for r in got]) for name in got[0]}


def _exact_distill(s):
    z, got = s["z"], []
    parts = _rows_at_once(z.shape[1])
    for part, ids, top, w in zip(*(s[n].split(parts) for n in ("z", "ids", "top", "weights"))):
        lq = torch.log_softmax(part.double() * s["scale"], 1)
        lp = torch.log_softmax(top.double() * s["scale"], 1)
        p, ids, w = lp.exp(), ids.long(), w.double()[:, None]
        row = {"loss": (w * p * (lp - torch.gather(lq, 1, ids))).sum(1)}
        if s["grad"]:
            target = torch.zeros_like(lq).scatter_(1, ids, p)
            # kept in 32 bits: 24 of the 53 are more than enough beside outputs of 8 or 24
            row["grad"] = ((lq.exp() - target) * w * s["scale"]).float()
        got.append(row)
    return {name: torch.cat([r[name] for r in got]) for name in got[0]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "logprobs": _exact_logprobs, "distill": _exact_distill}[case["op"]](s)
