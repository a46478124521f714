"""Calibrate the attention block of one decoder layer, keep its 8-bit codes, and serve requests with it.

    python examples/serve_layer.py [--config cfg4] [--requests 4] [--prompt 700] [--steps 16]

1. The scale search finds the input scale of the query/key/value projection (one matrix, one scale) on synthetic calibration
   activations; these go through the quantized projection, the cache and attention, and what comes out calibrates the output
   projection.  tlq_apply_layer gives the codes that are kept.
2. A step is: quantize the inputs -> tlq_linear_i8 -> tlq_kv_store (rotation, 8-bit cache) -> tlq_kv_attention -> quantize ->
   tlq_linear_i8.  All prompts go through it at once, then every request appends one token per step; that step is recorded
   once as a CUDA graph and replayed.
3. The outputs are compared with the same block in 32-bit floats: once on the values that the projections' codes stand for
   (what is left is the 8-bit cache and the rounding of attention's results), once without any quantization.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2602_07899_b200 import tlq, workloads as wl  # noqa: E402


class AttentionBlock:
    """Quantized query/key/value projection, 8-bit cache, attention and output projection of one layer."""

    def __init__(self, w_qkv, w_o, x, importance, cos_sin, n_heads, n_kv, head_dim):
        self.cfg = tlq.config(tlq.W8A8_SYM)
        self.n_heads, self.n_kv, self.head_dim = n_heads, n_kv, head_dim
        self.qkv = self._keep(w_qkv, x, importance)
        n, dev = x.shape[0], x.device
        blocks = -(-n // tlq.KV_BLOCK)
        cache = self.cache(blocks)
        batch = tlq.KvBatch(torch.tensor([0, n], dtype=torch.int32, device=dev), torch.tensor([n], dtype=torch.int32, device=dev),
                            torch.arange(blocks, dtype=torch.int32, device=dev)[None], n)
        ws = {"qkv": None, "kv": tlq.kv_workspace(cache, n_heads, n, batch)}
        self.o = self._keep(w_o, self._attend(x, cache, batch, torch.arange(n, dtype=torch.int32, device=dev), cos_sin, ws), importance)

    def _keep(self, w, x, importance):
        s = tlq.tlq_scale_search_layer(x, w, importance, self.cfg).s_best
        kept = tlq.tlq_apply_layer(x, w, s, None, self.cfg)
        return {"s": s, "codes": kept["codes"], "steps": kept["steps"]}

    def cache(self, n_blocks):
        return tlq.KvCache.empty(n_blocks, self.n_kv, self.head_dim, self.qkv["codes"].device)

    def workspaces(self, cache, batch, tokens):
        """Kept by the caller, one set per stream: zeroed once, good for any call of up to `tokens` tokens."""
        dev = self.qkv["codes"].device
        return {"qkv": tlq.linear_workspace(tokens, *reversed(self.qkv["codes"].shape), dev),
                "o": tlq.linear_workspace(tokens, *reversed(self.o["codes"].shape), dev),
                "kv": tlq.kv_workspace(cache, self.n_heads, tokens, batch)}

    def _attend(self, x, cache, batch, positions, cos_sin, ws):
        codes, steps = tlq.tlq_quantize_activations(x, self.qkv["s"], self.cfg)
        qkv = tlq.tlq_linear_i8(codes, steps, self.qkv["codes"], self.qkv["steps"], workspace=ws["qkv"])
        q, _, _ = tlq.tlq_kv_store(qkv, self.n_heads, cache, batch, positions, cos_sin, workspace=ws["kv"])
        y, _ = tlq.tlq_kv_attention(q, cache, batch, self.head_dim ** -0.5, workspace=ws["kv"])
        return y.flatten(1)

    def __call__(self, x, cache, batch, positions, cos_sin, ws):
        y = self._attend(x, cache, batch, positions, cos_sin, ws)
        codes, steps = tlq.tlq_quantize_activations(y, self.o["s"], self.cfg)
        return tlq.tlq_linear_i8(codes, steps, self.o["codes"], self.o["steps"], workspace=ws["o"])


def angles(n, head_dim, device):
    a = torch.outer(torch.arange(n, dtype=torch.float64), 1e6 ** (-torch.arange(head_dim // 2, dtype=torch.float64) / (head_dim // 2)))
    return torch.cat([a.cos(), a.sin()], 1).float().to(device)


def plain(x, w_qkv, w_o, s_o, n_heads, n_kv, d, cos_sin):
    """The block in 32 bits for one request whose tokens are all of x [n, hidden]; attention's results are divided by s_o."""
    n = x.shape[0]
    q, k, v = (x.float() @ w_qkv.float().t()).unflatten(1, (n_heads + 2 * n_kv, d)).split((n_heads, n_kv, n_kv), 1)
    c, s = cos_sin[:n, None, :d // 2], cos_sin[:n, None, d // 2:]

    def turn(z):
        a, b = z[..., :d // 2], z[..., d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    q, k = turn(q), turn(k).repeat_interleave(n_heads // n_kv, 1)
    v = v.repeat_interleave(n_heads // n_kv, 1)
    z = torch.einsum("qhd,khd->hqk", q, k) * d ** -0.5
    z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), float("-inf"))
    return (torch.einsum("hqk,khd->qhd", z.softmax(-1), v).flatten(1) / s_o) @ w_o.float().t()


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--config", default="cfg4", help="layer sizes (a key of the package's workloads)")
    p.add_argument("--requests", type=int, default=4)
    p.add_argument("--prompt", type=int, default=700, help="tokens of the longest prompt; the others are shorter")
    p.add_argument("--steps", type=int, default=16, help="tokens answered to every request")
    p.add_argument("--calibration", type=int, default=512, help="calibration tokens")
    a = p.parse_args(argv)
    dev, d = "cuda", 128
    c = wl.config(a.config, mode="w8a8")
    n_heads, n_kv = c.hidden // d, c.kv // d
    bits = lambda b: tlq.bf16_from_bits(b, dev)  # noqa: E731
    w_qkv = torch.cat([bits(wl.weights(c.seed, f"example/w_{n}", o, c.hidden)) for n, o in (("q", c.hidden), ("k", c.kv), ("v", c.kv))])
    w_o = bits(wl.weights(c.seed, "example/w_o", c.hidden, c.hidden))
    some = lambda name, n: bits(wl.activations(c.seed, "example/" + name, n, c.hidden, n // 2))  # noqa: E731
    imp = torch.from_numpy(wl.importance(c.seed, "example/w_imp", a.calibration, a.calibration // 2)).to(dev)
    # requests of different lengths, their blocks anywhere in the cache
    lens = [max(1, a.prompt * (r + 1) // a.requests - r) for r in range(a.requests)][::-1]
    need = [-(-(n + a.steps) // tlq.KV_BLOCK) for n in lens]
    order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).to(torch.int32).split(need)
    table = torch.zeros(a.requests, max(need), dtype=torch.int32)
    for r in range(a.requests):
        table[r, :need[r]] = order[r]
    table = table.to(dev)
    cos_sin = angles(max(max(lens) + a.steps, a.calibration), d, dev)
    block = AttentionBlock(w_qkv, w_o, some("x_attn_in", a.calibration), imp, cos_sin, n_heads, n_kv, d)
    cache = block.cache(sum(need))
    tokens = [some(f"request{r}", n + a.steps) for r, n in enumerate(lens)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731

    # the prompts
    x = torch.cat([t[:n] for t, n in zip(tokens, lens)])
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    batch = tlq.KvBatch(ints(starts), ints(lens), table, max(lens))
    ws = block.workspaces(cache, batch, x.shape[0])
    prompts = block(x, cache, batch, torch.cat([torch.arange(n) for n in lens]).to(torch.int32).to(dev), cos_sin, ws)
    outs = [[y] for y in prompts.split(lens)]

    # one token of every request per step, recorded once: only the inputs, lengths and positions change
    kv_len, pos = ints([n + 1 for n in lens]), ints(lens)
    batch = tlq.KvBatch(torch.arange(a.requests + 1, dtype=torch.int32, device=dev), kv_len, table, 1)
    x = torch.stack([t[n] for t, n in zip(tokens, lens)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x, cache, batch, pos, cos_sin, ws)              # storing a token twice leaves the cache as storing it once
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block(x, cache, batch, pos, cos_sin, ws)
    for i in range(a.steps):
        x.copy_(torch.stack([t[n + i] for t, n in zip(tokens, lens)]))
        graph.replay()
        for r in range(a.requests):
            outs[r].append(y[r:r + 1].clone())
        if i + 1 < a.steps:
            kv_len += 1
            pos += 1
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(50):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    for name, w in ws.items():
        status = tlq.tlq_read_status(w)
        if status != tlq.OK:
            raise RuntimeError(f"{name}: {tlq.status_string(status)}")

    worst = 0.0
    sizes = (n_heads, n_kv, d, cos_sin)
    stands_for = lambda kept: kept["codes"].float() * kept["steps"][:, None]  # noqa: E731
    for r, n in enumerate(lens):
        codes, steps = tlq.tlq_quantize_activations(tokens[r], block.qkv["s"], block.cfg)
        near = plain(codes.float() * steps[:, None], stands_for(block.qkv), stands_for(block.o), block.o["s"].float(), *sizes)
        whole, got = plain(tokens[r], w_qkv, w_o, 1.0, *sizes), torch.cat(outs[r]).float()
        for what, rows in (("prompt", slice(0, n)), ("answer", slice(n, None))):
            err, full = (float((got[rows] - w[rows]).norm() / w[rows].norm()) for w in (near, whole))
            worst = max(worst, err)
            print(f"request {r}: {what} of {got[rows].shape[0]} tokens, {100 * err:.2f} % from the codes' values, "
                  f"{100 * full:.2f} % from the unquantized block")
    print(f"one step of {a.requests} requests: {begin.elapsed_time(end) / 50 * 1e3:.0f} us")
    return worst


if __name__ == "__main__":
    main()
