"""The serving operators' definitions in 64 bits, on the CPU, as plain loops over requests and heads."""
import math

import torch

BLOCK = 64
FLOOR = 1e-5


def linear(xq, t, wq, u, bias):
    """-> (y, sum of the magnitudes that were added), float64."""
    acc = (xq.to(torch.int64).double() @ wq.to(torch.int64).double().t())
    y = acc * torch.outer(t.double(), u.double())
    mag = y.abs()
    if bias is not None:
        y = y + bias.double()
        mag = mag + bias.double().abs()
    return y, mag


def normed(x, w, eps):
    if w is None:
        return x
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()


def rotated(x, positions, sections, cos_sin):
    """x [T, heads, D] float64; positions [axes, T]."""
    if positions is None:
        return x
    half = x.shape[-1] // 2
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    c = torch.stack([cos_sin[positions[axis[i]].long(), i] for i in range(half)], 1).double()[:, None]
    s = torch.stack([cos_sin[positions[axis[i]].long(), half + i] for i in range(half)], 1).double()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def attention(q, kc, vc, ks, vs, cu, kv_len, table, scale, causal):
    """-> (out, lse, sum of p |v|, sum of |code| times the largest p * step of the row, largest magnitude of a score)
    float64, all [T, heads, ...]."""
    T, H, D = q.shape
    hk = kc.shape[1]
    out = torch.zeros(T, H, D, dtype=torch.float64)
    mag = torch.zeros(T, H, D, dtype=torch.float64)
    small = torch.zeros(T, H, D, dtype=torch.float64)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    weight = torch.zeros(T, H, dtype=torch.float64)
    for r in range(len(kv_len)):
        n, length = int(cu[r + 1] - cu[r]), int(kv_len[r])
        if n == 0 or length == 0:
            continue
        blocks = table[r, : -(-length // BLOCK)].long()
        seen = torch.arange(length)[None] <= (length - n + torch.arange(n))[:, None]
        for h in range(H):
            g = h // (H // hk)
            k = (kc[blocks, g].double() * ks[blocks, g].double()[:, None, None]).reshape(-1, D)[:length]
            v = (vc[blocks, g].double() * vs[blocks, g].double()[:, None, None]).transpose(1, 2).reshape(-1, D)[:length]
            x = q[int(cu[r]):int(cu[r + 1]), h].double()
            z = x @ k.t() * scale
            z_mag = (x.abs() @ k.abs().t() * scale).amax(1)
            if causal:
                z = torch.where(seen, z, torch.tensor(-math.inf, dtype=torch.float64))
            top = z.amax(1, keepdim=True)
            live = top[:, 0] > -math.inf
            p = torch.exp(z - torch.where(live[:, None], top, 0.0))
            total = p.sum(1, keepdim=True)
            rows = slice(int(cu[r]), int(cu[r + 1]))
            safe = torch.where(total > 0, total, 1.0)
            out[rows, h] = (p @ v) / safe
            mag[rows, h] = (p @ v.abs()) / safe
            steps = vs[blocks, g].double().repeat_interleave(BLOCK)[:length]
            codes = vc[blocks, g].double().transpose(1, 2).reshape(-1, D)[:length].abs()
            seen_too = (z > -math.inf).double()
            small[rows, h] = (p * steps).amax(1, keepdim=True) * (seen_too @ codes) / safe
            lse[rows, h] = torch.where(live, top[:, 0] + torch.log(safe[:, 0]), torch.tensor(-math.inf, dtype=torch.float64))
            weight[rows, h] = z_mag
    return out, lse, mag, small, weight
