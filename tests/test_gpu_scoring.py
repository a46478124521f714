"""Log probabilities with entropy and alternatives, and the distillation loss with its gradient, against their definitions in 64 bits, at
the sizes, masks and orders where they can go wrong."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
MASKED = -2.0 ** 100


@pytest.fixture(scope="module")
def tlq():
    from paper_2602_07899_b200 import tlq as mod
    return mod


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def logits_of(n, v, dtype, seed=0, spread=2.0):
    g = gen(seed + 7 * n + v)
    z = torch.randn(n, v, generator=g, device="cuda") * spread
    z[torch.arange(n, device="cuda"), torch.randint(0, v, (n,), generator=g, device="cuda")] += 9
    return z.to(dtype)


def masked64(z, scale):
    """scale z in 64 bits, masked logits as -infinity."""
    return torch.where(z.double() <= MASKED, -math.inf, z.double() * scale)


def from_top(a):
    """(a less its row's largest, the logarithm of the sum of their exponentials, the largest): far from zero 64 bits keep no more."""
    top = a.amax(1, keepdim=True)
    top = torch.where(torch.isinf(top) & (top < 0), 0.0, top)
    return a - top, (a - top).exp().sum(1, keepdim=True).log(), top


def slack(v):
    """Of the logarithm of a sum: one rounding of 2^-24 for each addition in a row (a thread's share of the row is v / 512, or v / 128 of
    rows up to 32 KB, and 30 to join them), 2^-21 of the exponential, and 30 2^-23 of its argument (terms further down than 30 are below
    2^-30 of the sum)."""
    return (max(v / 512, min(v, 16384) / 128) + 30) * 2.0 ** -24 + 2.0 ** -21 + 30 * 2.0 ** -23


def order_of(z, k):
    """The k largest, the lower index first among equals; masked logits are equals."""
    z = torch.where(z.float() <= MASKED, MASKED, z.float())
    return torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]


def check_logprobs(tlq, z, ids, k, scale=1.0):
    n, v = z.shape
    out = tlq.tlq_token_logprobs(z, ids, k, scale, want_entropy=True, want_lse=True)
    a = masked64(z, scale)
    d, total, largest = from_top(a)
    lse = (largest + total)[:, 0]
    lp = torch.where(torch.isinf(a), a, d - total)
    none = torch.isinf(lse)
    most = slack(v)
    assert torch.equal(torch.isinf(out["lse"]) & (out["lse"] < 0), none)
    assert torch.all((out["lse"].double() - lse).abs()[~none] <= most + 2.0 ** -22 * lse.abs()[~none])

    def close(got, want):           # log probabilities: the scale's rounding on top, 2^-23 of them
        inf = torch.isinf(want) | torch.isnan(want)
        assert torch.all(got[inf] == -math.inf)
        assert torch.all((got.double() - want).abs()[~inf] <= most + 2.0 ** -22 * want.abs()[~inf])
    if ids is not None:
        given = (ids >= 0) & (ids < v)
        assert torch.all(out["logp"][ids < 0] == 0) and torch.isnan(out["logp"][ids >= v]).all()
        close(out["logp"][given], lp[given].gather(1, ids[given].long()[:, None])[:, 0])
    p = lp.exp().nan_to_num(0.0)
    weight = (p * lp.abs().nan_to_num(posinf=0.0, neginf=0.0)).sum(1)        # (the entropy: each term off by the same parts)
    assert torch.all(out["entropy"][none] == 0)
    assert torch.all((out["entropy"].double() - weight).abs() <= 2 * most * (1 + weight + total[:, 0].nan_to_num(neginf=0.0).abs()))
    if k:
        top = order_of(z, k)
        have = top.shape[1]
        assert torch.equal(out["top_ids"][:, :have].long(), top)
        close(out["top_logp"][:, :have], lp.gather(1, top))
        assert torch.all(out["top_ids"][:, have:] == -1) and torch.all(out["top_logp"][:, have:] == -math.inf)
    return out


def some_ids(n, v, seed=0):
    ids = torch.randint(0, v, (n,), generator=gen(seed), device="cuda").to(I32)
    ids[::5] = -1
    ids[1::7] = v - 1
    ids[2::11] = v
    ids[3::13] = 0
    return ids


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 31, 100, 129, 1000, 1024, 4097, 8191, 16384, 16385, 16391, 50001, 131072, 262147])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_logprobs_over_sizes(tlq, n, v, dtype):
    z = logits_of(n, v, dtype)
    for k, scale in ((0, 1.0), (1, 0.5), (20, 1.25), (128, 1.0)):
        check_logprobs(tlq, z, some_ids(n, v), k, scale)


@pytest.mark.parametrize("n,v,dtype", [(1000, 1000, BF16), (3000, 33, F32), (700, 20011, BF16), (600, 40000, F32), (20000, 7, BF16)])
def test_logprobs_of_many_rows(tlq, n, v, dtype):
    check_logprobs(tlq, logits_of(n, v, dtype), some_ids(n, v), 64)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v,pitch", [(1001, 1008), (50257, 50304), (131072, 131075), (77, 1000)])
def test_logprobs_of_strided_rows_at_any_alignment(tlq, v, pitch, dtype):
    n = 9
    wide = torch.full((n, pitch + 11), math.nan, dtype=dtype, device="cuda")
    for at in (0, 1, 3, 6, 11 if pitch >= v + 11 else 2):
        z = wide[:, at:at + v]
        z.copy_(logits_of(n, v, dtype, at))
        check_logprobs(tlq, z, some_ids(n, v), 20)
        z.fill_(math.nan)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [9, 1000, 16385, 131072])
def test_logprobs_of_masked_rows(tlq, v, dtype):
    z = logits_of(8, v, dtype)
    z[0] = -math.inf                                    # nothing left
    z[1, 1:] = -math.inf                                # the first one left
    z[2, :-1] = torch.finfo(dtype).min                  # the last one left, masked by the type's lowest value
    z[3, ::2] = -math.inf
    z[4, 3:] = -1e31
    z[5] = torch.finfo(dtype).min
    z[6, v // 2:] = -math.inf
    ids = torch.tensor([0, 0, v - 1, 0, 1, 2, v - 1, -1], dtype=I32, device="cuda")
    for k in (1, 5, 64, 128):
        check_logprobs(tlq, z, ids, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [100, 4096, 50001, 131072])
def test_alternatives_of_equal_logits_come_by_index(tlq, v, dtype):
    n = 6
    z = torch.zeros(n, v, dtype=dtype, device="cuda")
    z[1] = torch.randint(-2, 3, (v,), generator=gen(1), device="cuda").to(dtype)
    z[2, 1::2] = -0.0                                   # equal to 0
    z[3] = -5
    z[4] = torch.randint(0, 2, (v,), generator=gen(2), device="cuda").to(dtype) * -math.inf
    z[4].nan_to_num_(nan=0.0, neginf=-math.inf)
    z[5, v // 3] = 1
    for k in (1, 20, 128):
        check_logprobs(tlq, z, None, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v", [(13, 300), (13, 8000), (13, 131072), (700, 20011), (1, 262147)])
def test_alternatives_of_rows_with_few_or_crowded_tokens(tlq, n, v, dtype):
    """All masked but some, side by side or strewn about: those come first, then the first of the masked ones."""
    g = gen(v)
    z = torch.randn(n, v, generator=g, device="cuda").to(dtype)
    index = torch.arange(v, device="cuda")
    allowed = torch.zeros(n, v, dtype=torch.bool, device="cuda")
    for i, count in enumerate((0, 1, 5, 19, 20, 21, 63, 64, 65, 128, 129, 1000, 2000)):
        for j in range(i, n, 13):
            count = min(count, v)
            start = (0, v - count, (v - count) // 2 + 3)[j % 3] if count < v - 8 else 0
            allowed[j] = (index >= start) & (index < start + count)
            if j % 4 == 3:
                allowed[j] = allowed[j, torch.randperm(v, generator=g, device="cuda")]
    z = torch.where(allowed, z, torch.tensor(-math.inf if v % 2 else -1e38, dtype=dtype, device="cuda"))
    for k in (1, 20, 64, 128):
        check_logprobs(tlq, z, None, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [5000, 131072])
def test_alternatives_in_orders_that_defeat_a_bound(tlq, v, dtype):
    """Rising and falling rows, and rows whose large logits all belong to a few threads: more of them than there is room for."""
    i = torch.arange(v, device="cuda")
    vec = 16 // torch.finfo(dtype).bits * 8
    rows = [i / v * 8, -i / v * 8, torch.where(i // vec % 512 < 60, 4.0, 0.0) + i % 97 / 64, torch.where(i // vec % 128 < 60, 4.0, 0.0) + i % 97 / 64,
            torch.where(i < v // 2, 3.0, 0.0) + (i * 7919 % v) / v, torch.where(i // vec % 512 == 5, 4.0, 0.0) + (i * 31 % 1009) / 512]
    z = torch.stack([r.float() for r in rows]).to(dtype)
    for k in (1, 63, 64, 128):
        check_logprobs(tlq, z, None, k)
        check_logprobs(tlq, z.repeat(120, 1)[:700], None, k)            # a row to a CTA


@pytest.mark.parametrize("v", [77, 50001, 131072])
def test_rows_that_are_not_numbers_have_no_distribution(tlq, v):
    for dtype in (BF16, F32):
        z = logits_of(7, v, dtype)
        clean = tlq.tlq_token_logprobs(z, some_ids(7, v), 20, want_entropy=True, want_lse=True)
        bad = z.clone()
        bad[0, v - 1], bad[3, 5], bad[5, 0] = math.nan, math.inf, -math.nan
        out = tlq.tlq_token_logprobs(bad, torch.zeros(7, dtype=I32, device="cuda"), 20, want_entropy=True, want_lse=True)
        hit = [0, 3, 5]
        for name in ("logp", "entropy", "lse", "top_logp"):
            assert torch.isnan(out[name][hit]).all()
        assert torch.all(out["top_ids"][hit] == -1)
        rest = [1, 2, 4, 6]
        for name in ("entropy", "lse", "top_ids", "top_logp"):
            assert torch.equal(out[name][rest], clean[name][rest])


def test_logprobs_of_large_logits_and_extreme_scales(tlq):
    z = logits_of(5, 40000, F32, spread=3000.0)
    check_logprobs(tlq, z, some_ids(5, 40000), 20)
    check_logprobs(tlq, z, some_ids(5, 40000), 20, 2.0 ** -16)
    check_logprobs(tlq, logits_of(5, 40000, F32), some_ids(5, 40000), 20, 2.0 ** 16)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [100, 4096, 50001, 131072])
def test_logprobs_and_distillation_of_rows_far_from_zero(tlq, v, dtype):
    """Rows of one value, as an added mask leaves them, from -1e30 to 1e38: an even distribution; and rows of a few values out there."""
    n = 12
    z = torch.empty(n, v, dtype=F32, device="cuda")
    for r, x in enumerate((-1e30, -1e25, -1e9, -3e8, 1e9, 1e20, 2e38)):
        z[r] = x
    z[7] = -1e30
    z[7, 5:9] = -1e9
    z[8] = -1e30
    z[8, v // 2] = -0.5e30
    z[9] = 1e9
    z[9, 3::7] = 1.5e9
    z[10, :] = -1e9
    z[10, 0] = 4.0
    z[11] = torch.randn(v, generator=gen(1), device="cuda") - 2.0 ** 20
    z = z.to(dtype)
    scales = (1.0, 0.5, 2.0 ** -16)
    for scale in scales:
        check_logprobs(tlq, z, some_ids(n, v), 20, scale)
        ids, top = teacher_of(z, 20)
        check_distill(tlq, z, ids, torch.where(top.abs() > 1e37, top / 1e8, top), None, scale)
    check_logprobs(tlq, z[:6].contiguous(), None, 128, 2.0 ** 16)


def test_each_output_alone_is_what_it_is_among_the_others(tlq):
    z, ids = logits_of(33, 30000, BF16), some_ids(33, 30000)
    every = tlq.tlq_token_logprobs(z, ids, 10, want_entropy=True, want_lse=True)
    assert torch.equal(tlq.tlq_token_logprobs(z, ids)["logp"].nan_to_num(7.0), every["logp"].nan_to_num(7.0))
    assert torch.equal(tlq.tlq_token_logprobs(z, want_lse=True)["lse"], every["lse"])
    assert torch.equal(tlq.tlq_token_logprobs(z, want_entropy=True)["entropy"], every["entropy"])
    assert torch.equal(tlq.tlq_token_logprobs(z, top_k=10)["top_logp"], every["top_logp"])


def test_logprobs_beyond_four_billion_bytes(tlq):
    n, v = 17000, 131072
    z = torch.zeros(n, v, dtype=BF16, device="cuda")
    last = logits_of(3, v, BF16)
    z[-3:] = last
    out = tlq.tlq_token_logprobs(z, None, 8, want_entropy=True, want_lse=True)
    want = tlq.tlq_token_logprobs(last, None, 8, want_entropy=True, want_lse=True)
    assert torch.equal(out["top_ids"][-3:], want["top_ids"])
    assert torch.all((out["lse"][-3:] - want["lse"]).abs() <= 2 * slack(v) + 2.0 ** -22 * want["lse"].abs())
    assert torch.all((out["lse"][:-3] - math.log(v)).abs() <= 2 * slack(v) + 2.0 ** -21 * math.log(v))


# ---------------------------------------------------------------------------------------------- distillation

def distill_ref(z, ids, top, w, scale):
    """(loss, gradient, p, q of each row's teacher) in 64 bits, place by place."""
    a = masked64(z, scale)
    d, total, _ = from_top(a)
    lse, lp = total, torch.where(torch.isinf(a), a, d - total)       # (lse: -infinity where nothing is left)
    given = ids >= 0
    t = torch.where(given & (top.double() > MASKED), top.double() * scale, -math.inf)
    has = (t > -math.inf).any(1)
    dt, total_t, _ = from_top(t)
    lt = torch.where(torch.isinf(t), t, dt - total_t)
    p = torch.where(has[:, None], lt.exp(), 0.0)
    at = ids.long().clamp(0, z.shape[1] - 1)
    lq = lp.gather(1, at)       # (a masked token has no probability, of whatever is left)
    terms = torch.where(p > 0, p * (lt - lq), 0.0)
    w = torch.ones(len(z), dtype=torch.float64, device=z.device) if w is None else w.double()
    loss = torch.where(has & (w != 0), w * terms.sum(1), 0.0)
    q = torch.where(torch.isinf(lse), 0.0, lp.exp())
    target = torch.zeros_like(q).scatter_add_(1, at, p)
    alive = has & (w != 0) & ~torch.isinf(lse[:, 0])
    grad = torch.where(alive[:, None], (w * scale)[:, None] * (q - target), 0.0)
    size = torch.where(alive[:, None], (w.abs() * scale)[:, None] * (q + target), 0.0)
    return loss, grad, size, (p * (lt.nan_to_num(neginf=0.0).abs() + lq.abs().nan_to_num(posinf=0.0))).sum(1) * w.abs()


def check_distill(tlq, z, ids, top, w, scale=1.0, grad=None):
    loss, want, size, mag = distill_ref(z, ids, top, w, scale)
    v, dtype = z.shape[1], z.dtype
    most = slack(v)
    alone, none = tlq.tlq_distill_loss(z, ids, top, w, scale, want_grad=False)
    assert none is None
    got, g = tlq.tlq_distill_loss(z, ids, top, w, scale, grad=grad)
    weight = torch.ones_like(loss) if w is None else w.double().abs()
    inf = torch.isinf(loss)
    assert torch.equal(torch.isinf(got) & (got > 0), inf)
    assert torch.all((got.double() - loss).abs()[~inf] <= (weight * 2 * most + 4 * most * mag)[~inf] + 2.0 ** -23 * loss.abs()[~inf])
    # (without the gradient a row may be shared by another number of CTAs: the same bound)
    assert torch.all((alone.double() - loss).abs()[~inf] <= (weight * 2 * most + 4 * most * mag)[~inf] + 2.0 ** -23 * loss.abs()[~inf])
    # q and p are off by the slack of their logarithm, each of its own size; then one rounding
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert g.dtype == dtype and g.shape == z.shape
    assert torch.all((g.double() - want).abs() <= half * (want.abs() + 4 * most * size) + 4 * most * size + 2.0 ** -126)
    return got, g


def teacher_of(z, k, seed=0):
    t = z.float() + 0.7 * torch.randn(z.shape, generator=gen(seed), device="cuda")
    top, ids = torch.topk(t, k, dim=1)
    return ids.to(I32).contiguous(), top.contiguous()


def weights_of(n, seed=3):
    w = torch.exp(torch.randn(n, generator=gen(seed), device="cuda"))
    w[1::4] = 0
    return w


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [1, 2, 9, 31, 129, 1000, 4097, 16391, 50001, 131072, 262147])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_distill_over_sizes(tlq, n, v, dtype):
    z = logits_of(n, v, dtype)
    for k, scale, w in ((1, 1.0, None), (20, 0.5, weights_of(n)), (128, 1.25, weights_of(n))):
        ids, top = teacher_of(z, min(k, v))
        check_distill(tlq, z, ids, top, w, scale)


@pytest.mark.parametrize("n,v,dtype", [(1000, 1000, BF16), (2000, 33, F32), (700, 20011, BF16), (400, 40000, F32), (600, 65537, BF16)])
def test_distill_of_many_rows(tlq, n, v, dtype):
    z = logits_of(n, v, dtype)
    check_distill(tlq, z, *teacher_of(z, 20), weights_of(n))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v,pitch", [(1001, 1008), (50257, 50304), (77, 1000)])
def test_distill_of_strided_rows_at_any_alignment_and_in_place(tlq, v, pitch, dtype):
    n = 9
    wide, out = (torch.full((n, pitch + 11), 5.0, dtype=dtype, device="cuda") for _ in range(2))
    for at, to in ((0, 0), (1, 0), (3, 3), (6, 2)):
        z, g = wide[:, at:at + v], out[:, to:to + v]
        z.copy_(logits_of(n, v, dtype, at))
        ids, top = teacher_of(z, 20)
        _, a = check_distill(tlq, z, ids, top, weights_of(n))
        out.fill_(5.0)
        _, b = check_distill(tlq, z, ids, top, weights_of(n), grad=g)
        assert b is g and torch.equal(a, b)
        assert torch.all(out[:, :to] == 5) and torch.all(out[:, to + v:] == 5)
        loss, c = tlq.tlq_distill_loss(z, ids, top, weights_of(n), grad=z)
        assert torch.equal(c, a) and torch.all(wide[:, :at] == 5) and torch.all(wide[:, at + v:] == 5)
        wide.fill_(5.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v,pitch,start", [(6, 1, 3, 1), (6, 5, 9, 2), (40, 77, 80, 3), (700, 1000, 1001, 1), (5, 4090, 4099, 6), (5, 8193, 8200, 0),
                                             (700, 20011, 20012, 5), (600, 65537, 65544, 0), (3, 262147, 262150, 7)])
def test_distill_gradient_that_lies_elsewhere_on_the_grid_than_the_logits(tlq, n, v, pitch, start, dtype):
    """Rows of the gradient at all offsets from those of the logits: the same gradient bit for bit, and nothing beside it touched."""
    z = logits_of(n, v, dtype)
    ids, top = teacher_of(z, min(v, 7))
    w = weights_of(n)
    w[1::3] = 0.0
    loss, want = tlq.tlq_distill_loss(z, ids, top, w)
    buf = torch.full((n * pitch + 16,), 7.0, dtype=dtype, device="cuda")
    grad = buf[start:start + n * pitch].view(n, pitch)[:, :v]
    again, _ = tlq.tlq_distill_loss(z, ids, top, w, grad=grad)
    assert torch.equal(again, loss) and torch.equal(grad, want)
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[start:start + n * pitch].view(n, pitch)[:, :v] = False
    assert torch.all(buf[rest] == 7)


def test_distill_in_place_with_a_row_over_several_ctas(tlq):
    for n, v, dtype in ((1, 262147, F32), (5, 131072, BF16), (300, 131072, BF16)):
        z = logits_of(n, v, dtype)
        ids, top = teacher_of(z, 64)
        loss, g = tlq.tlq_distill_loss(z, ids, top)
        again, h = tlq.tlq_distill_loss(z, ids, top, grad=z)
        assert torch.equal(loss, again) and torch.equal(g, h)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [50, 50001])
def test_distill_of_places_that_are_empty_repeated_or_masked(tlq, v, dtype):
    n, k = 9, 20
    z = logits_of(n, v, dtype)
    ids, top = teacher_of(z, k)
    ids[0] = -1                             # no teacher
    top[1] = -math.inf                      # no teacher either
    ids[2, 5:] = -3                         # some places
    ids[3] = ids[3, 0]                      # one token in every place
    ids[4, 1::2] = ids[4, ::2]              # pairs
    top[5, 3:] = torch.finfo(F32).min       # teacher's masked
    z[6, ids[6, 0].long()] = -math.inf      # the student's is masked where the teacher's is not: an infinite loss
    z[7] = -math.inf                        # nothing left of the student
    top[8, 1:] = top[8, :1]
    check_distill(tlq, z, ids, top, None)
    check_distill(tlq, z, ids, top, weights_of(n) + 0.5, 0.5)


@pytest.mark.parametrize("v", [60, 131072])
def test_distill_keeps_what_is_no_number_to_its_row(tlq, v):
    for dtype in (BF16, F32):
        z = logits_of(8, v, dtype)
        ids, top = teacher_of(z, 20)
        w = torch.ones(8, device="cuda")
        w[[3, 4]] = 0
        clean, g0 = tlq.tlq_distill_loss(z, ids, top, w)
        bad, ids2, top2 = z.clone(), ids.clone(), top.clone()
        bad[0, 7], bad[1, v - 1], bad[3] = math.nan, math.inf, math.nan       # (row 3 does not count)
        ids2[2, 4], ids2[4, 0] = v, v + 7                                    # ids outside of the vocabulary; row 4 does not count
        top2[5, 0] = math.nan
        loss, g = tlq.tlq_distill_loss(bad, ids2, top2, w)
        assert torch.isnan(loss[[0, 1, 2, 5]]).all() and torch.all(loss[[3, 4]] == 0)
        assert torch.isnan(g[[0, 1, 2]].float()).all() and torch.all(g[[3, 4]] == 0)
        assert torch.isnan(g[5].float().gather(0, ids2[5].long())).all()
        assert torch.equal(loss[[6, 7]], clean[[6, 7]]) and torch.equal(g[[6, 7]], g0[[6, 7]])


def test_distill_gradient_against_differences(tlq):
    """Central differences of the loss (of 64 bits: 32 leave nothing of them), and the sum over a row, which is 0."""
    n, v, k, scale = 4, 40, 6, 0.75
    z = logits_of(n, v, F32)
    ids, top = teacher_of(z, k)
    ids[1, 3] = ids[1, 0]
    w = torch.tensor([1.0, 2.5, -0.5, 0.3], device="cuda")
    _, g = tlq.tlq_distill_loss(z, ids, top, w, scale)
    assert torch.all(g.double().sum(1).abs() <= 2.0 ** -18 * w.double().abs())
    for c in range(v):
        e = torch.zeros(v, dtype=torch.float64, device="cuda")
        e[c] = 1e-4
        d = (distill_ref(z.double() + e, ids, top, w, scale)[0] - distill_ref(z.double() - e, ids, top, w, scale)[0]) / 2e-4
        # the third derivative of ln q is below 1: (1e-4)^2 / 6 of it, and 2^-52 / 1e-4 of losses of up to 40
        assert torch.all((g[:, c].double() - d).abs() <= 2e-9 + 2.0 ** -44 / 1e-4 + 2.0 ** -18 * w.double().abs())


@pytest.mark.parametrize("n,v,dtype", [(600, 65537, BF16), (400, 40000, F32), (300, 131072, BF16), (2000, 9000, BF16)])
def test_scoring_gives_the_same_in_call_after_call(tlq, n, v, dtype):
    """Slots that are filled again while others still read would show here, now and then."""
    z = logits_of(n, v, dtype)
    ids, top = teacher_of(z, 20)
    w = weights_of(n)
    first = (*tlq.tlq_distill_loss(z, ids, top, w), *tlq.tlq_token_logprobs(z, None, 64, want_entropy=True, want_lse=True).values())
    for rep in range(60):
        if rep % 2:
            tlq.tlq_distill_loss(z, ids, top, w, want_grad=False)
        again = (*tlq.tlq_distill_loss(z, ids, top, w), *tlq.tlq_token_logprobs(z, None, 64, want_entropy=True, want_lse=True).values())
        assert all(a is None or torch.equal(a, b) for a, b in zip(first, again))


FIRST_CALL = '''
import torch
from paper_2602_07899_b200 import tlq
x = torch.randn(300, 4096, device="cuda").bfloat16()
big = torch.randn(40, 70000, device="cuda").bfloat16()
ids = torch.zeros(300, 4, dtype=torch.int32, device="cuda")
top = torch.randn(300, 4, device="cuda")
def calls():
    n = tlq.tlq_norm_quantize(x, None, want_values=True)
    w = torch.ones(4096, 4096, dtype=torch.int8, device="cuda")
    u = torch.ones(4096, device="cuda")
    p = tlq.tlq_linear_i8_act(n["codes"], n["steps"], w, u, act=1, gated=True)
    return [n["codes"], n["values"], p, *tlq.tlq_token_logprobs(x, ids[:, 0].contiguous(), 5, want_entropy=True).values(), *tlq.tlq_token_logprobs(big, None, 5).values(),
            *tlq.tlq_distill_loss(x, ids, top), *tlq.tlq_distill_loss(big, ids[:40].contiguous(), top[:40].contiguous())]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    a = calls()
graph.replay()
b = calls()
torch.cuda.synchronize()
assert all(s is None or torch.equal(s, t) for s, t in zip(a, b))
print("same")
'''


def test_first_calls_of_a_process_can_be_recorded(tlq):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_scoring_repeats_bit_for_bit_on_another_stream_and_in_a_graph(tlq):
    for n, v, dtype in ((1, 131072, BF16), (64, 50001, F32), (900, 20011, BF16)):
        z, ids = logits_of(n, v, dtype), some_ids(n, v)
        tid, top = teacher_of(z, 64)

        def both(stream=None):
            r = tlq.tlq_token_logprobs(z, ids, 64, want_entropy=True, want_lse=True, stream=stream)
            loss, grad = tlq.tlq_distill_loss(z, tid, top, stream=stream)
            return [v.view(torch.int32) if v.dtype == F32 else v for v in (*r.values(), loss, grad)]
        a = both()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        b = both(side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c = both()
        for t in c:
            t.zero_()
        graph.replay()
        assert all(torch.equal(x, y) and torch.equal(x, w) for x, y, w in zip(a, b, c))


def test_distill_gradient_beyond_four_billion_bytes(tlq):
    n, v = 17000, 131072
    z = torch.zeros(n, v, dtype=BF16, device="cuda")
    last = logits_of(3, v, BF16)
    z[-3:] = last
    ids, top = teacher_of(last, 8)
    ids, top = (torch.cat([t[:1].expand(n - 3, -1), t]).contiguous() for t in (ids, top))
    ids[:n - 3, 1:] = -1
    loss, g = tlq.tlq_distill_loss(z, ids, top, grad=z)
    want, h = tlq.tlq_distill_loss(last, ids[-3:].contiguous(), top[-3:].contiguous())
    assert g is z and torch.all((loss[-3:] - want).abs() <= 4 * slack(v) * (1 + want.abs()))
    assert torch.all((g[-3:].float() - h.float()).abs() <= 2.0 ** -7 * h.float().abs() + 4 * slack(v) * h.float().abs())
    assert torch.all((loss[:-3] - math.log(v)).abs() <= 4 * slack(v) * math.log(v))
    rest = g[1000:1003].double()
    at = ids[0, 0].long()
    assert torch.all((rest[:, at] + 1).abs() <= 2.0 ** -8)
    rest[:, at] = 1 / v
    assert torch.all((rest - 1 / v).abs() <= (2.0 ** -8 + 4 * slack(v)) / v)


def test_scoring_of_no_rows(tlq):
    z = torch.zeros(0, 100, dtype=BF16, device="cuda")
    assert tlq.tlq_token_logprobs(z, torch.zeros(0, dtype=I32, device="cuda"), 5)["top_ids"].shape == (0, 5)
    loss, g = tlq.tlq_distill_loss(z, torch.zeros(0, 4, dtype=I32, device="cuda"), torch.zeros(0, 4, device="cuda"))
    assert loss.shape == (0,) and g.shape == (0, 100)


def test_from_a_teachers_alternatives_to_the_importance_of_tokens(tlq):
    """The full-precision model's alternatives are the teacher's logits of the quantized one, whose gradient weighs the tokens."""
    n, c, v = 96, 512, 4096
    g = gen(9)
    x = torch.randn(n, c, generator=g, device="cuda").bfloat16()
    head = (torch.randn(v, c, generator=g, device="cuda") * 4 * c ** -0.5).bfloat16()
    cfg = tlq.config(tlq.W8A8_SYM)
    kept = tlq.tlq_quantize_weights(head, None, cfg)
    first = tlq.tlq_norm_quantize(x, None, cfg, want_y=True)
    teacher = (first["y"].float() @ head.float().t())
    student = tlq.tlq_linear_i8(first["codes"], first["steps"], kept["codes"], kept["steps"])
    best = check_logprobs(tlq, teacher, None, 32)
    score = check_logprobs(tlq, student, best["top_ids"][:, 0].contiguous(), 0)
    assert float((score["logp"] - best["top_logp"][:, 0]).abs().mean()) < 0.1
    loss, grad = check_distill(tlq, student, best["top_ids"], best["top_logp"], None)
    imp, mask = tlq.tlq_token_importance(grad[None], tlq.NORM_L2, 0.5)
    want = grad.double().norm(dim=1)
    assert torch.all((imp.double() - want).abs() <= 1e-5 * want) and int(mask.sum()) == n // 2
    # these weights go where the calibration takes the importance of tokens
    best_scale = tlq.tlq_scale_search_layer(first["y"], head, imp, cfg)
    assert 0 <= int(best_scale.best_idx) < cfg.n_grid


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [1000, 4093])
def test_importance_from_a_teacher(tlq, v, dtype):
    from paper_2602_07899_b200 import calibrate
    n = 60
    z = logits_of(n, v, dtype)
    ids, top = teacher_of(z, 20)
    w = weights_of(n)
    loss, grad = tlq.tlq_distill_loss(z, ids, top, w)
    for kind, norm in ((tlq.NORM_L2, grad.double().norm(dim=1)), (tlq.NORM_MEAN_ABS, grad.double().abs().mean(1))):
        imp, mask, got = calibrate.importance_from_teacher(z, ids, top, w, norm_kind=kind)
        assert torch.equal(got, loss) and int(mask.sum()) == n // 2
        assert torch.all((imp.double() - norm).abs() <= 1e-5 * norm)          # (an fp32 result of fp64 sums of fp32 parts)
        assert float(imp[mask.bool()].min()) >= float(imp[~mask.bool()].max())
