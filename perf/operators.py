"""The serving operators of a calibrated decoder layer, as cases that can be measured: the 8-bit product, the norm /
rotation / 8-bit cache write of queries, keys and values, and attention over that cache.

Every operator has its plain form here (elementary torch operations in 32 bits, rounded once at the end) and, with
`own` set, the calls that a user makes of this package.  Sizes: the 7B-, 72B- and 2B-class layers of the package's
workloads (hidden 3584 / 8192 / 1536, key-value width 512 / 1024 / 256, heads of 128 channels) and a small layer with
heads of 64 channels.
"""
import math
import random

import torch

own = False

BLOCK = 64          # tokens of one cache block
FLOOR = 1e-5        # smallest |.| maximum that a quantization step is made from
EPS = 1e-6

# heads of queries, heads of keys and values, channels of a head
HEADS = {"7b": (28, 4, 128), "72b": (64, 8, 128), "2b": (12, 2, 128), "small": (14, 2, 64), "equal": (8, 8, 64)}


def listed():
    return [
        # one token of a chat through the smallest projection of the 7B-class layer: launch latency
        {"name": "linear: 1 token, key projection", "op": "linear", "tokens": 1, "c_in": 3584, "c_out": 512, "bias": True},
        # a decoding batch of 16 chats through the widest weights: the weights' bytes
        {"name": "linear: 16 tokens, gate", "op": "linear", "tokens": 16, "c_in": 3584, "c_out": 18944, "bias": False},
        # a short prompt (odd length) through the 2B-class gate
        {"name": "linear: 201 tokens, 2B gate", "op": "linear", "tokens": 201, "c_in": 1536, "c_out": 8960, "bias": True},
        # a calibration batch, or a long prompt, through the 7B-class gate: the tensor cores
        {"name": "linear: 8192 tokens, gate", "op": "linear", "tokens": 8192, "c_in": 3584, "c_out": 18944, "bias": False},
        # one decoding step of 32 chats: every request appends one token somewhere inside a block
        {"name": "store: 32 requests, 1 token", "op": "store", "model": "7b", "requests": 32, "q_max": 1, "kv_max": 5000,
         "ragged": True, "norm": False, "axes": 3, "lens": 1},
        # prompts of several chats with images (three position axes), some continuing inside a block
        {"name": "store: 6 ragged prompts", "op": "store", "model": "2b", "requests": 6, "q_max": 1501, "kv_max": 2900,
         "ragged": True, "norm": True, "axes": 3, "lens": 2},
        # one long prompt of the 72B-class layer: bytes in and out
        {"name": "store: 16384 token prompt", "op": "store", "model": "72b", "requests": 1, "q_max": 16384, "kv_max": 16384,
         "ragged": False, "norm": True, "axes": 1, "lens": 3},
        # the first answers of one chat: latency
        {"name": "attention: 1 token over 100", "op": "attention", "model": "2b", "requests": 1, "q_max": 1, "kv_max": 100,
         "ragged": False, "causal": True, "lens": 4},
        # a decoding step of 64 chats of very different age: the cache's bytes, unevenly split
        {"name": "attention: 64 requests, 1 token", "op": "attention", "model": "7b", "requests": 64, "q_max": 1,
         "kv_max": 32761, "ragged": True, "causal": True, "lens": 5},
        # one token over a very long context: the work has to be split over the context
        {"name": "attention: 1 token over 131071", "op": "attention", "model": "72b", "requests": 1, "q_max": 1,
         "kv_max": 131071, "ragged": False, "causal": True, "lens": 6},
        # chunks of prompts over contexts already in the cache, of different lengths
        {"name": "attention: 3 ragged chunks", "op": "attention", "model": "7b", "requests": 3, "q_max": 511, "kv_max": 16001,
         "ragged": True, "causal": True, "lens": 7},
        # a whole prompt: the tensor cores
        {"name": "attention: 8192 token prompt", "op": "attention", "model": "7b", "requests": 1, "q_max": 8192, "kv_max": 8192,
         "ragged": False, "causal": True, "lens": 8},
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(("linear", "linear", "store", "attention", "attention", "attention"))
    if op == "linear":
        c_in = 16 * _log(rng, 8, 1184)
        c_in += 16 if c_in == 3072 else 0
        c_out = _log(rng, 200, 18944)
        most = 8192 * 3584 * 18944 // (c_in * c_out)
        return {"op": op, "tokens": _log(rng, 1, min(8192, most)), "c_in": c_in, "c_out": c_out, "bias": rng.random() < 0.5}
    model = rng.choice(sorted(HEADS))
    case = {"op": op, "model": model, "ragged": rng.random() < 0.7, "lens": rng.randrange(1 << 20)}
    if op == "store":
        n = _log(rng, 1, 64)
        q = 1 if rng.random() < 0.3 else _log(rng, 2, 16384 // n)
        return {**case, "requests": n, "q_max": q, "kv_max": _log(rng, q, 16384), "norm": rng.random() < 0.5,
                "axes": rng.choice((1, 3))}
    heads = HEADS[model][0]
    if rng.random() < 0.5:      # decoding, or a few drafted tokens at once
        n = _log(rng, 1, 64)
        q = rng.choice((1, 1, 1, 2, 5))
        kv = _log(rng, q, min(131072, 32761 * 64 * 4 // (n * HEADS[model][1])))
    else:
        n = _log(rng, 1, 6)
        kv = _log(rng, 16, 16384)
        q = _log(rng, 1, min(kv, max(1, 8192 * 8192 * 28 // (2 * n * kv * heads))))
    return {**case, "requests": n, "q_max": q, "kv_max": kv, "causal": rng.random() < 0.8}


# ------------------------------------------------------------------------------------------------ lengths

def _lens(case):
    """(new tokens, cached tokens after them) of every request, from the case alone."""
    n, q_max, kv_max = case["requests"], case["q_max"], case["kv_max"]
    if not case["ragged"]:
        return [q_max] * n, [kv_max] * n
    rng = random.Random(case["lens"])
    q, kv = [q_max], [kv_max]
    for _ in range(n - 1):
        q.append(_log(rng, 1, q_max))
        kv.append(max(q[-1], _log(rng, 1, kv_max)))
    if n >= 4:                  # a slot of the batch that has nothing to do in this step
        q[-1] = 0
    return q, kv


def _visible(case):
    """Pairs of a query and a key that it sees, over all requests."""
    total = 0
    for q, kv in zip(*_lens(case)):
        total += q * kv - (q * (q - 1) // 2 if case["causal"] else 0)
    return total


def work(case):
    if case["op"] == "linear":
        n, ci, co = case["tokens"], case["c_in"], case["c_out"]
        return {"bytes": n * ci + ci * co + 4 * (n + co) + (2 * co if case["bias"] else 0) + 2 * n * co, "flops": 2 * n * ci * co}
    hq, hk, d = HEADS[case["model"]]
    q, kv = _lens(case)
    tokens = sum(q)
    if case["op"] == "store":
        touched = sum(-(-k // BLOCK) - (k - n) // BLOCK for n, k in zip(q, kv) if n)
        # queries, keys, values in; queries out, codes and the values they stand for out; positions, angles, steps
        moved = tokens * d * (2 * (hq + 2 * hk) + 2 * hq + 2 * hk + 4 * hk) + tokens * (4 * case["axes"] + 4 * d) + 16 * touched * hk
        return {"bytes": moved, "flops": tokens * d * (8 * hq + 12 * hk)}
    moved = 2 * sum(k for n, k in zip(q, kv) if n) * hk * d + tokens * hq * (4 * d + 4)
    moved += 8 * hk * sum(-(-k // BLOCK) for n, k in zip(q, kv) if n)
    return {"bytes": moved, "flops": 4 * d * hq * _visible(case)}


# ------------------------------------------------------------------------------------------------ inputs

def _codes(x, dim):
    """int8 codes and the step of x over the dimensions `dim`."""
    step = x.abs().amax(dim, keepdim=True).clamp_min(FLOOR) / 127
    return torch.round(x / step).to(torch.int8), step


def _linear_inputs(case, g, dev):
    n, ci, co = case["tokens"], case["c_in"], case["c_out"]
    x = torch.randn(n, ci, generator=g, device=dev)
    x[:, torch.randint(0, ci, (4,), generator=g, device=dev)] *= 8      # activations keep a few large channels
    xq, t = _codes(x, 1)
    wq, u = _codes(torch.randn(co, ci, generator=g, device=dev) * 0.02, 1)
    bias = torch.randn(co, generator=g, device=dev).bfloat16() if case["bias"] else None
    return {"xq": xq, "t": t.flatten().contiguous(), "wq": wq, "u": u.flatten().contiguous(), "bias": bias}


def _batch_inputs(case, g, dev):
    """Lengths, a shuffled block table and a cache filled as earlier steps leave it."""
    hq, hk, d = HEADS[case["model"]]
    q, kv = _lens(case)
    need = [-(-k // BLOCK) for k in kv]
    n_blocks, width = sum(need) + 3, max(need)
    order = torch.randperm(n_blocks, generator=g, device=dev).to(torch.int32)
    first = torch.tensor([sum(need[:i]) for i in range(len(need))], device=dev)
    col = torch.arange(width, device=dev)
    table = order[(first[:, None] + col).clamp_max(n_blocks - 1)]
    table = torch.where(col < torch.tensor(need, device=dev)[:, None], table, 0).to(torch.int32).contiguous()
    k = torch.randn(n_blocks, hk, BLOCK, d, generator=g, device=dev)
    k[..., torch.randint(0, d, (2,), generator=g, device=dev)] *= 4     # keys have channels of their own size
    kc, ks = _codes(k, (2, 3))
    del k
    vc, vs = _codes(torch.randn(n_blocks, hk, d, BLOCK, generator=g, device=dev), (2, 3))   # values lie channel by token
    cu = [0]
    for n in q:
        cu.append(cu[-1] + n)
    return {"kc": kc, "vc": vc, "ks": ks.reshape(n_blocks, hk).contiguous(), "vs": vs.reshape(n_blocks, hk).contiguous(),
            "cu": torch.tensor(cu, dtype=torch.int32, device=dev), "kv": torch.tensor(kv, dtype=torch.int32, device=dev),
            "table": table, "tokens": cu[-1], "q_max": max(q), "hq": hq, "hk": hk, "d": d}


def _sections(d, axes):
    """Rotation pairs of each position axis: time, height, width."""
    if axes == 1:
        return (d // 2,)
    third = 3 * d // 16
    return (d // 2 - 2 * third, third, third)


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    if case["op"] == "linear":
        s = _linear_inputs(case, g, dev)
        tokens, width = case["tokens"], case["c_out"]
    else:
        s = _batch_inputs(case, g, dev)
        tokens, d = s["tokens"], s["d"]
        if case["op"] == "store":
            axes = case["axes"]
            s["qkv"] = torch.randn(tokens, (s["hq"] + 2 * s["hk"]) * d, generator=g, device=dev).bfloat16()
            limit = case["kv_max"] + 64
            angle = torch.outer(torch.arange(limit, device=dev, dtype=torch.float64),
                                1e6 ** (-torch.arange(d // 2, device=dev, dtype=torch.float64) / (d // 2)))
            s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
            s["positions"] = torch.randint(0, limit, (axes, tokens), generator=g, device=dev).to(torch.int32)
            s["sections"] = _sections(d, axes)
            s["qw"] = s["kw"] = None
            if case["norm"]:
                s["qw"] = (1 + 0.2 * torch.randn(d, generator=g, device=dev)).bfloat16()
                s["kw"] = (1 + 0.2 * torch.randn(d, generator=g, device=dev)).bfloat16()
        else:
            s["q"] = (1.5 * torch.randn(tokens, s["hq"], d, generator=g, device=dev)).bfloat16()
            s["scale"], s["causal"] = d ** -0.5, case["causal"]
    s["op"] = case["op"]
    if own:     # what a serving program makes once: the handle of its cache, the batch's lengths, a workspace
        from paper_2602_07899_b200 import tlq
        s["tlq"] = tlq
        if case["op"] == "linear":
            s["ws"] = tlq.linear_workspace(tokens, case["c_in"], width, dev)
        else:
            s["cache"] = tlq.KvCache(s["kc"], s["vc"], s["ks"], s["vs"])
            s["batch"] = tlq.KvBatch(s["cu"], s["kv"], s["table"], s["q_max"])
            s["ws"] = tlq.kv_workspace(s["cache"], s["hq"], tokens, s["batch"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_linear(s):
    y = (s["xq"].float() @ s["wq"].float().t()) * s["t"][:, None] * s["u"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.bfloat16()


def _places(s):
    """Of every new token: its request, its number in it and its place in the request's context."""
    token = torch.arange(s["tokens"], device=s["cu"].device)
    cu, kv = s["cu"].long(), s["kv"].long()
    req = torch.searchsorted(cu, token, right=True) - 1
    i = token - cu[req]
    return req, i, kv[req] - (cu[1:] - cu[:-1])[req] + i


def _norm(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _rotate(x, s):
    half = s["d"] // 2
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=x.device),
                                   torch.tensor(s["sections"], device=x.device), output_size=half)
    at = s["positions"].long()[axis].t()                                # [tokens, half]
    pair = torch.arange(half, device=x.device)
    c, n = s["cos_sin"][at, pair][:, None], s["cos_sin"][at, pair + half][:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * n, b * c + a * n], -1)


def _write(x, codes, steps, first, start, fresh, phys, off, channel_major):
    """Quantize x [tokens, heads, channels] into its blocks; the values that the new codes stand for."""
    n_blocks, hk = steps.shape
    top = x.abs().amax(-1)
    top = torch.zeros(n_blocks, hk, device=x.device).index_reduce_(0, phys, top, "amax")
    new = torch.zeros(n_blocks, dtype=torch.bool, device=x.device).index_fill_(0, phys, True)[:, None]
    old = torch.where(fresh[:, None], torch.zeros_like(steps), steps)
    step = torch.where(new, torch.maximum(old, top.clamp_min(FLOOR) / 127), steps)
    # tokens already in a request's first block follow a step that grew
    ratio = torch.where(new & (old > 0), old / step, torch.ones_like(step))[first]
    held = codes[first].float()
    moved = torch.round(held * ratio[:, :, None, None])
    place = torch.arange(BLOCK, device=x.device)
    inside = (place < start[:, None])[:, None]
    inside = inside[:, :, None, :] if channel_major else inside[:, :, :, None]
    codes[first] = torch.where(inside, moved, held).to(torch.int8)
    c = torch.round(x / step[phys][..., None]).clamp(-127, 127)
    if channel_major:
        codes[phys, :, :, off] = c.to(torch.int8)
    else:
        codes[phys, :, off] = c.to(torch.int8)
    steps.copy_(step)
    return (c * step[phys][..., None]).bfloat16()


def _plain_store(s):
    hq, hk, d = s["hq"], s["hk"], s["d"]
    x = s["qkv"].float().view(s["tokens"], hq + 2 * hk, d)
    q = _rotate(_norm(x[:, :hq], s["qw"]), s)
    k = _rotate(_norm(x[:, hq:hq + hk], s["kw"]), s)
    v = x[:, hq + hk:]
    req, _, place = _places(s)
    table, kv, cu = s["table"].long(), s["kv"].long(), s["cu"].long()
    phys, off = table[req, place // BLOCK], place % BLOCK
    begin = kv - (cu[1:] - cu[:-1])
    first = table.gather(1, (begin // BLOCK).clamp_max(table.shape[1] - 1)[:, None])[:, 0]
    # a block whose first token is written now holds nothing that counts
    fresh = torch.zeros(len(s["ks"]), dtype=torch.int32, device=x.device).index_add_(0, phys, (off == 0).int()) > 0
    start = torch.where((begin % BLOCK > 0) & (cu[1:] > cu[:-1]), begin % BLOCK, 0)
    kval = _write(k, s["kc"], s["ks"], first, start, fresh, phys, off, False)
    vval = _write(v, s["vc"], s["vs"], first, start, fresh, phys, off, True)
    return {"q": q.bfloat16(), "k": kval, "v": vval, "k_steps": s["ks"], "v_steps": s["vs"]}


def _plain_attention(s):
    hq, hk, d, n = s["hq"], s["hk"], s["d"], len(s["kv"])
    group, dev = hq // hk, s["q"].device
    table, kv, cu = s["table"].long(), s["kv"].long(), s["cu"].long()
    k = s["kc"][table].float().mul_(s["ks"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(n, hk, -1, d)
    v = s["vc"][table].float().mul_(s["vs"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(n, hk, -1, d)
    row, key = torch.arange(s["q_max"], device=dev), torch.arange(k.shape[2], device=dev)
    q = s["q"].float()[(cu[:-1, None] + row).clamp_max(s["tokens"] - 1)]               # [requests, q_max, heads, channels]
    q = q.view(n, -1, hk, group, d).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, d)
    score = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(n, hk, group, -1, k.shape[2])
    last = kv[:, None] - 1 + row * 0
    if s["causal"]:
        last = torch.minimum(last, (kv - (cu[1:] - cu[:-1]))[:, None] + row)
    score.masked_fill_((key > last[:, :, None])[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(n, hk, -1, k.shape[2]) @ v).view(n, hk, group, -1, d) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + total.log())[..., 0]
    req, i, _ = _places(s)
    return {"out": out[req, :, :, i].reshape(-1, hq, d).bfloat16(), "lse": lse[req, :, :, i].reshape(-1, hq)}


def run(s):
    if own:
        t = s["tlq"]
        if s["op"] == "linear":
            return t.tlq_linear_i8(s["xq"], s["t"], s["wq"], s["u"], s["bias"], workspace=s["ws"])
        if s["op"] == "store":
            q, k, v = t.tlq_kv_store(s["qkv"], s["hq"], s["cache"], s["batch"], s["positions"], s["cos_sin"], s["sections"],
                                     s["qw"], s["kw"], EPS, want_values=True, workspace=s["ws"])
            return {"q": q, "k": k, "v": v, "k_steps": s["ks"], "v_steps": s["vs"]}
        out, lse = t.tlq_kv_attention(s["q"], s["cache"], s["batch"], s["scale"], s["causal"], want_lse=True, workspace=s["ws"])
        return {"out": out, "lse": lse}
    return {"linear": _plain_linear, "store": _plain_store, "attention": _plain_attention}[s["op"]](s)


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_store(s):
    """Request by request and block by block, as the definition reads."""
    hq, hk, d = s["hq"], s["hk"], s["d"]
    half = d // 2
    x = s["qkv"].double().view(-1, hq + 2 * hk, d)
    angle_c, angle_s = s["cos_sin"].double()[:, :half], s["cos_sin"].double()[:, half:]
    pos = s["positions"].long()
    cs, sn, at = [], [], 0
    for axis, count in enumerate(s["sections"]):
        cs.append(angle_c[pos[axis], at:at + count])
        sn.append(angle_s[pos[axis], at:at + count])
        at += count
    cs, sn = torch.cat(cs, 1)[:, None], torch.cat(sn, 1)[:, None]

    def turned(y, w):
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
        return torch.cat([y[..., :half] * cs - y[..., half:] * sn, y[..., half:] * cs + y[..., :half] * sn], -1)

    q, new = turned(x[:, :hq], s["qw"]), {"k": turned(x[:, hq:hq + hk], s["kw"]), "v": x[:, hq + hk:]}
    steps = {"k": s["ks"].double().clone(), "v": s["vs"].double().clone()}
    vals = {"k": torch.empty_like(new["k"]), "v": torch.empty_like(new["k"])}
    cu, kv, table = s["cu"].tolist(), s["kv"].tolist(), s["table"].tolist()
    for r in range(len(kv)):
        place, token = kv[r] - (cu[r + 1] - cu[r]), cu[r]
        while token < cu[r + 1]:
            take = min(BLOCK - place % BLOCK, cu[r + 1] - token)
            block = table[r][place // BLOCK]
            for name in ("k", "v"):
                part = new[name][token:token + take]
                step = part.abs().amax((0, 2)).clamp_min(FLOOR) / 127
                if place % BLOCK:
                    step = torch.maximum(step, steps[name][block])
                steps[name][block] = step
                vals[name][token:token + take] = torch.round(part / step[:, None]) * step[:, None]
            token, place = token + take, place + take
    return {"q": q, "k": vals["k"], "v": vals["v"], "k_steps": steps["k"], "v_steps": steps["v"]}


def _exact_attention(s):
    """Request by request and head by head."""
    hq, hk, d = s["hq"], s["hk"], s["d"]
    cu, kv, table = s["cu"].tolist(), s["kv"].tolist(), s["table"].long()
    out = torch.zeros(s["tokens"], hq, d, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((s["tokens"], hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for r in range(len(kv)):
        n, length = cu[r + 1] - cu[r], kv[r]
        if n == 0 or length == 0:
            continue
        blocks = table[r, :-(-length // BLOCK)]
        seen = torch.arange(length, device=out.device)[None] <= (length - n + torch.arange(n, device=out.device))[:, None]
        for h in range(hk):
            k = (s["kc"][blocks, h].double() * s["ks"].double()[blocks, h, None, None]).reshape(-1, d)[:length]
            v = (s["vc"][blocks, h].double() * s["vs"].double()[blocks, h, None, None]).transpose(1, 2).reshape(-1, d)[:length]
            for j in range(h * (hq // hk), (h + 1) * (hq // hk)):
                z = s["q"][cu[r]:cu[r + 1], j].double() @ k.t() * s["scale"]
                if s["causal"]:
                    z = torch.where(seen, z, -math.inf)
                lse[cu[r]:cu[r + 1], j] = torch.logsumexp(z, 1)
                out[cu[r]:cu[r + 1], j] = torch.softmax(z, 1) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        y = torch.mm(s["xq"].double(), s["wq"].double().t())
        y = y * torch.outer(s["t"].double(), s["u"].double())
        return y if s["bias"] is None else y + s["bias"].double()
    return _exact_store(s) if case["op"] == "store" else _exact_attention(s)
