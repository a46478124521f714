"""The serving operators against their definitions in 64 bits: the 8-bit product, the key-value store (norm, rotation,
8-bit cache write) and attention over the 8-bit cache, at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

BLOCK = 64


@pytest.fixture(scope="module")
def tlq():
    from paper_2602_07899_b200 import tlq as mod
    return mod


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---------------------------------------------------------------------------------------------- 8-bit product

def linear_case(n, ci, co, bias, seed=0):
    g = gen(seed + n * 7 + ci * 3 + co)
    xq = torch.randint(-127, 128, (n, ci), generator=g).to(torch.int8)
    wq = torch.randint(-128, 128, (co, ci), generator=g).to(torch.int8)
    t = torch.rand(n, generator=g) * 0.05 + 1e-4
    u = torch.rand(co, generator=g) * 0.002 + 1e-6
    b = torch.randn(co, generator=g).bfloat16() if bias else None
    return xq, t, wq, u, b


def linear_close(y, want, mag):
    """One rounding to bf16 (8 significant bits: 2^-8 of the value) after four roundings to fp32."""
    err = (y.double().cpu() - want).abs()
    assert torch.all(err <= 2.0 ** -8 * want.abs() * (1 + 2.0 ** -7) + 2.0 ** -21 * mag)


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 100, 127, 128, 129, 200, 256, 257, 515, 1031])
@pytest.mark.parametrize("ci,co", [(16, 1), (48, 17), (208, 130), (1040, 264), (3584, 512)])
def test_linear_small_shapes(tlq, n, ci, co):
    xq, t, wq, u, b = linear_case(n, ci, co, (n + co) % 2 == 0)
    want, mag = ref.linear(xq, t, wq, u, b)
    y = tlq.tlq_linear_i8(xq.cuda(), t.cuda(), wq.cuda(), u.cuda(), None if b is None else b.cuda())
    linear_close(y, want, mag)


@pytest.mark.parametrize("n,ci,co", [(1, 18944, 3584), (3, 29568, 1024), (12, 8192, 1000), (40, 18944, 515), (300, 8960, 1536),
                                     (2048, 1536, 8960), (1000, 131056, 24)])
def test_linear_layer_shapes(tlq, n, ci, co):
    xq, t, wq, u, b = linear_case(n, ci, co, True)
    # 64-bit product on the device: integers below 2^53 are exact
    acc = xq.cuda().double() @ wq.cuda().double().t()
    want = acc * torch.outer(t.cuda().double(), u.cuda().double())
    mag = (want.abs() + b.cuda().double().abs()).cpu()
    want = (want + b.cuda().double()).cpu()
    y = tlq.tlq_linear_i8(xq.cuda(), t.cuda(), wq.cuda(), u.cuda(), b.cuda())
    linear_close(y, want, mag)


@pytest.mark.parametrize("n,ci,co", [(1, 3584, 512), (5, 4096, 100), (48, 4096, 256), (130, 4096, 257), (512, 2048, 512)])
def test_linear_sums_are_exact_integers(tlq, n, ci, co):
    """Extreme codes: every sum is the largest there is; with steps of a power of two the result is the rounded integer."""
    xq = torch.full((n, ci), -128, dtype=torch.int8)
    xq[:, ::3] = 127
    wq = torch.full((co, ci), -128, dtype=torch.int8)
    wq[::2, 1::5] = 127
    one = torch.ones
    y = tlq.tlq_linear_i8(xq.cuda(), one(n).cuda(), wq.cuda(), (one(co) * 2.0 ** -10).cuda())
    acc = (xq.double() @ wq.double().t()) * 2.0 ** -10
    assert torch.equal(y.cpu(), acc.float().bfloat16())


def test_linear_repeats_bit_for_bit_and_on_another_stream(tlq):
    for n in (4, 24, 150, 700):
        xq, t, wq, u, b = [v.cuda() for v in linear_case(n, 3584, 512, True)]
        ws = tlq.linear_workspace(n, 3584, 512, "cuda")
        y = tlq.tlq_linear_i8(xq, t, wq, u, b, workspace=ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            z = [tlq.tlq_linear_i8(xq, t, wq, u, b, workspace=ws) for _ in range(3)]
        side.synchronize()
        assert all(torch.equal(y, w) for w in z)
        assert tlq.tlq_read_status(ws) == tlq.OK


def test_linear_of_no_tokens(tlq):
    xq, t, wq, u, b = linear_case(0, 64, 32, True)
    y = tlq.tlq_linear_i8(xq.cuda(), t.cuda(), wq.cuda(), u.cuda(), b.cuda())
    assert y.shape == (0, 32)


def test_linear_of_quantized_codes_is_apply_layer(tlq):
    """From the calibration's own codes: the same layer as tlq_apply_layer (which quantizes on every call)."""
    g = gen(3)
    X = torch.randn(70, 512, generator=g).bfloat16().cuda()
    W = (torch.randn(264, 512, generator=g) * 0.02).bfloat16().cuda()
    bias = torch.randn(264, generator=g).bfloat16().cuda()
    s = (torch.rand(512, generator=g) + 0.5).bfloat16().cuda()
    cfg = tlq.config(tlq.W8A8_SYM)
    whole = tlq.tlq_apply_layer(X, W, s, bias, cfg)
    xq, t = tlq.tlq_quantize_activations(X, s, cfg)
    y = tlq.tlq_linear_i8(xq, t, whole["codes"], whole["steps"], bias)
    d = (y.float() - whole["Yq"].float()).abs()
    assert torch.all(d <= 2.0 ** -7 * whole["Yq"].float().abs())      # at most one unit of the last place


# ---------------------------------------------------------------------------------------------- batches

def make_batch(seed, q_lens, kv_lens, hk, d, extra=2, pad=1):
    """Shuffled blocks, table entries beyond a request's need that must not be read, codes in every place."""
    g = gen(seed)
    need = [-(-k // BLOCK) for k in kv_lens]
    n_blocks = sum(need) + extra
    order = torch.randperm(n_blocks, generator=g).to(torch.int32)
    table = torch.full((len(kv_lens), max(need + [1]) + pad), -7, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    kc = torch.randint(-127, 128, (n_blocks, hk, BLOCK, d), generator=g).to(torch.int8)
    vc = torch.randint(-127, 128, (n_blocks, hk, d, BLOCK), generator=g).to(torch.int8)
    ks = torch.rand(n_blocks, hk, generator=g) * 0.02 + 0.005
    vs = torch.exp(2 * torch.randn(n_blocks, hk, generator=g)) * 0.01
    unused = order[at:].long()
    ks[unused] = math.nan
    vs[unused] = math.inf
    cu = torch.tensor([0] + list(torch.tensor(q_lens).cumsum(0)), dtype=torch.int32)
    return dict(kc=kc, vc=vc, ks=ks, vs=vs, cu=cu, kv=torch.tensor(kv_lens, dtype=torch.int32), table=table, T=sum(q_lens),
                q_max=max(q_lens))


def on_gpu(tlq, s):
    cache = tlq.KvCache(s["kc"].cuda(), s["vc"].cuda(), s["ks"].cuda(), s["vs"].cuda())
    return cache, tlq.KvBatch(s["cu"].cuda(), s["kv"].cuda(), s["table"].cuda(), s["q_max"])


# ---------------------------------------------------------------------------------------------- attention

HEADS = [(12, 2, 128), (7, 1, 128), (8, 8, 64), (64, 8, 128), (14, 2, 64), (5, 1, 64), (32, 1, 128), (3, 3, 128)]
LENS = {
    "one token": ([1], [1]),
    "one token, 100 cached": ([1], [100]),
    "block edges": ([1, 1, 1, 1, 1, 1], [1, 63, 64, 65, 128, 129]),
    "idle slots": ([1, 0, 1, 0], [0, 70, 1, 0]),
    "long and short": ([1, 1, 1], [5000, 3, 700]),
    "drafts": ([2, 5, 3, 1], [2, 64, 131, 700]),
    "prompts": ([40, 1, 129, 64, 0], [40, 65, 500, 64, 9]),
    "chunk over context": ([65, 200], [777, 200]),
    "tokens before the first": ([5, 3], [3, 0]),
    "tile edges": ([127, 128, 129], [127, 300, 385]),
}


def attention_bounds(want, lse, mag, small, weight, d):
    """Scores are fp32 sums of d exact products (error d 2^-23 of their magnitudes, and the rounding of the scale and of the
    two logarithms); probabilities are rounded to 11 bits, or to 2^-36 of the row's largest p * step where that is more
    (the smallest 16-bit float is 2^-24, the largest p is kept at 2^11 at least); the output to 8."""
    ds = weight * (d * 2.0 ** -23) + 2.0 ** -19 * (1 + lse.abs().nan_to_num(posinf=0.0, neginf=0.0))
    rel = (2.0 ** -11 + 2.0 ** -18 + 2 * ds)[..., None]
    return 2.0 ** -8 * want.abs() * (1 + 2.0 ** -7) + rel * mag * 1.01 + 2.0 ** -36 * small + 1e-30, 2 * ds


def check_attention(tlq, s, heads, hk, d, causal, seed, stride=0):
    g = gen(seed)
    q = (torch.randn(s["T"], heads, d, generator=g) * 1.5).bfloat16()
    scale = d ** -0.5
    want, lse, mag, small, weight = ref.attention(q, s["kc"], s["vc"], s["ks"], s["vs"], s["cu"], s["kv"], s["table"], scale, causal)
    cache, batch = on_gpu(tlq, s)
    if stride:
        wide = torch.full((s["T"], heads * d + stride), math.nan, dtype=torch.bfloat16, device="cuda")
        wide[:, :heads * d] = q.cuda().reshape(s["T"], -1)
        qd = wide[:, :heads * d].unflatten(1, (heads, d))
    else:
        qd = q.cuda()
    ws = tlq.kv_workspace(cache, heads, s["T"], batch)
    for _ in range(2):                          # the second call finds the workspace as the first left it
        out, got = tlq.tlq_kv_attention(qd, cache, batch, scale, causal, want_lse=True, workspace=ws)
        assert tlq.tlq_read_status(ws) == tlq.OK
        most, most_lse = attention_bounds(want, lse, mag, small, weight, d)
        err = (out.double().cpu() - want).abs()
        assert torch.all(err <= most), float((err - most).max())
        none = torch.isinf(lse)
        got = got.double().cpu()
        assert torch.equal(torch.isinf(got) & (got < 0), none)
        assert torch.all((got - lse).abs()[~none] <= most_lse[~none])
        assert torch.all(out.cpu()[none] == 0)


# A request of this size takes a batch over the 3 M pairs from which requests of many rows have a kernel of their own.
BIG = (1000, 1400)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,hk,d", [(12, 2, 128), (7, 1, 128), (8, 8, 64), (14, 2, 64), (5, 1, 64), (32, 1, 128), (4, 4, 128)])
def test_attention_of_prompts(tlq, heads, hk, d, causal):
    """Row tiles and blocks that end anywhere, requests on both sides of the limit of rows, some of them empty."""
    q_lens, kv_lens = [40, 1, 129, 0, BIG[0], 64, 3, 257], [40, 65, 500, 9, BIG[1], 64, 0, 250]
    check_attention(tlq, make_batch(12, q_lens, kv_lens, hk, d), heads, hk, d, causal, 5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", sorted(LENS))
@pytest.mark.parametrize("heads,hk,d", HEADS)
def test_attention(tlq, heads, hk, d, lens, causal):
    q_lens, kv_lens = LENS[lens]
    check_attention(tlq, make_batch(11, q_lens, kv_lens, hk, d), heads, hk, d, causal, 5)


@pytest.mark.parametrize("heads,hk,d", [(28, 4, 128), (14, 2, 64)])
def test_attention_of_strided_queries(tlq, heads, hk, d):
    for q_lens, kv_lens in (([1, 1], [90, 200]), ([70, 200], [100, 260])):
        check_attention(tlq, make_batch(2, q_lens, kv_lens, hk, d), heads, hk, d, True, 6, stride=2 * hk * d)
    check_attention(tlq, make_batch(2, [70, BIG[0]], [100, BIG[1]], hk, d), heads, hk, d, True, 6, stride=2 * hk * d)


def test_attention_of_many_requests(tlq):
    g = gen(4)
    kv = [int(v) for v in torch.randint(0, 300, (700,), generator=g)]
    q = [1 if k else 0 for k in kv]
    check_attention(tlq, make_batch(5, q, kv, 1, 64), 4, 1, 64, True, 8)


@pytest.mark.parametrize("q_lens,kv_lens", [([1], [20000]), ([1, 1, 1], [9000, 1, 64]), ([130], [6000]), ([300, 1], [4500, 4500])])
def test_attention_split_over_the_context(tlq, q_lens, kv_lens):
    check_attention(tlq, make_batch(9, q_lens, kv_lens, 2, 128), 12, 2, 128, True, 10)


def test_attention_of_many_rows_before_the_first_key(tlq):
    """Runs of row tiles without a visible key between tiles that have some, several of both for every CTA."""
    check_attention(tlq, make_batch(19, [2000] * 20, [70] * 20, 8, 64), 8, 8, 64, True, 13)


@pytest.mark.parametrize("q_len,big", [(1, False), (150, False), (150, True)])
def test_attention_with_steps_of_zero_and_of_very_different_size(tlq, q_len, big):
    """A block of zeros (step 0) still takes part in the softmax; value steps span fourteen powers of ten."""
    s = make_batch(21, [q_len] + [BIG[0]] * big, [64 * 8] + [BIG[1]] * big, 1, 128)
    b = s["table"][0].long()
    s["ks"][b[1]] = 0.0
    s["vs"][b[2]] = 0.0
    s["vs"][b[3]] = 1e-9
    s["vs"][b[4]] = 1e5
    check_attention(tlq, s, 7, 1, 128, True, 3)
    check_attention(tlq, s, 7, 1, 128, False, 3)


@pytest.mark.parametrize("q_len,big", [(1, False), (150, False), (150, True)])
def test_attention_with_large_and_small_scores(tlq, q_len, big):
    """Scores in the hundreds either way: the running maximum moves far from block to block."""
    s = make_batch(22, [q_len] + [BIG[0]] * big, [64 * 9 + 5] + [BIG[1]] * big, 1, 64)
    b = s["table"][0].long()
    for i in range(9):
        s["ks"][b[i]] = (0.5, 0.0001, 0.02)[i % 3] * (i + 1)
    check_attention(tlq, s, 4, 1, 64, True, 4)


@pytest.mark.parametrize("q_len,big", [(1, False), (200, False), (200, True)])
def test_attention_keeps_non_finite_queries_to_their_rows(tlq, q_len, big):
    s = make_batch(31, [q_len, q_len] + [BIG[0]] * big, [400, 300] + [BIG[1]] * big, 2, 128)
    q = torch.randn(s["T"], 12, 128, generator=gen(1)).bfloat16()
    bad = q.clone()
    bad[0, 3, 5] = math.nan
    bad[q_len, 7, 9] = math.inf
    cache, batch = on_gpu(tlq, s)
    clean, _ = tlq.tlq_kv_attention(q.cuda(), cache, batch, 0.1)
    out, lse = tlq.tlq_kv_attention(bad.cuda(), cache, batch, 0.1, want_lse=True)
    hit = torch.zeros(s["T"], 12, dtype=torch.bool)
    hit[0, 3] = hit[q_len, 7] = True
    assert torch.equal(out.cpu()[~hit], clean.cpu()[~hit])
    assert torch.isnan(out.cpu()[0, 3]).all() and torch.isfinite(out.cpu()[~hit].float()).all()
    assert torch.isfinite(lse.cpu()[~hit]).all()


@pytest.mark.parametrize("q_len,kv_len", [(4, 200), BIG])
def test_attention_of_huge_and_tiny_queries(tlq, q_len, kv_len):
    """Rows far outside of the 16-bit float range of the products: a power of two per row takes care of them."""
    s = make_batch(33, [q_len], [kv_len], 1, 128)
    s["ks"][:] = s["ks"].nan_to_num(0.01) * 0 + 1e-3
    q = torch.randn(q_len, 7, 128, generator=gen(2)).bfloat16()
    cache, batch = on_gpu(tlq, s)
    want, _ = tlq.tlq_kv_attention(q.cuda(), cache, batch, 2.0 ** -3)
    for f in (2.0 ** 40, 2.0 ** -40, 2.0 ** -100):
        got, _ = tlq.tlq_kv_attention((q.float() * f).bfloat16().cuda(), cache, batch, 2.0 ** -3 / f)
        assert torch.equal(got, want)


def test_attention_of_prompts_reports_a_block_that_does_not_fit(tlq):
    s = make_batch(43, [BIG[0], 70], [BIG[1], 130], 1, 64)
    q = torch.randn(s["T"], 4, 64, generator=gen(3)).bfloat16().cuda()
    cache, batch = on_gpu(tlq, s)
    ws = tlq.kv_workspace(cache, 4, s["T"], batch)
    good, _ = tlq.tlq_kv_attention(q, cache, batch, 0.125, workspace=ws)
    assert tlq.tlq_read_status(ws) == tlq.OK
    s["table"][0, 3] = 1 << 30
    cache, batch = on_gpu(tlq, s)
    ws = tlq.kv_workspace(cache, 4, s["T"], batch)
    out, _ = tlq.tlq_kv_attention(q, cache, batch, 0.125, workspace=ws)
    assert tlq.tlq_read_status(ws) == tlq.ERR_SHAPE
    assert torch.equal(out[BIG[0]:], good[BIG[0]:]) and torch.isfinite(out.float()).all()


def test_attention_reports_metadata_that_does_not_fit(tlq):
    """A block outside of the cache, a length beyond the table: reported, left out, and the other requests unharmed."""
    q_lens, kv_lens = [1, 1, 70], [150, 200, 130]
    s = make_batch(41, q_lens, kv_lens, 1, 64)
    q = torch.randn(s["T"], 4, 64, generator=gen(3)).bfloat16().cuda()
    cache, batch = on_gpu(tlq, s)
    ws = tlq.kv_workspace(cache, 4, s["T"], batch)
    good, _ = tlq.tlq_kv_attention(q, cache, batch, 0.125, workspace=ws)
    assert tlq.tlq_read_status(ws) == tlq.OK
    for what in ("block", "length", "rows"):
        t = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
        if what == "block":
            t["table"][1, 1] = 1 << 30
        elif what == "length":
            t["kv"][1] = 1 << 30
            t["table"][1] = t["table"][1].clamp_min(0)
        else:
            t["cu"][3] = 1 << 20
        cache, batch = on_gpu(tlq, t)
        ws = tlq.kv_workspace(cache, 4, s["T"], batch)
        out, _ = tlq.tlq_kv_attention(q, cache, batch, 0.125, workspace=ws)
        assert tlq.tlq_read_status(ws) == tlq.ERR_SHAPE
        # the rest is split anew: the same values up to the rounding of probabilities and results
        for rows in (slice(0, 1), slice(2, None)):
            a, b = out[rows].float(), good[rows].float()
            assert torch.all((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -9 * b.abs().max())


# ---------------------------------------------------------------------------------------------- key-value store

def rope_table(n, d):
    ang = torch.outer(torch.arange(n, dtype=torch.float64), 1e4 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2)))
    return torch.cat([ang.cos(), ang.sin()], 1).float()


STORE_LENS = {
    "one token": ([1], [1]),
    "block edges": ([1, 1, 1, 1, 1], [1, 64, 65, 63, 200]),
    "idle slots": ([0, 1, 0], [70, 9, 0]),
    "prompts": ([40, 64, 129, 1, 65], [40, 64, 129, 70, 128]),
    "continued inside a block": ([3, 100, 64], [50, 130, 90]),
    "long": ([700], [1000]),
}


def run_store(tlq, s, heads, hk, d, norm, axes, seed, stride=0, qkv=None):
    g = gen(seed)
    width = (heads + 2 * hk) * d
    if qkv is None:
        qkv = (torch.randn(s["T"], width, generator=g) * 2).bfloat16()
    table = rope_table(1500, d)
    pos = torch.randint(0, 1500, (axes, s["T"]), generator=g).to(torch.int32) if axes else None
    sections = {0: None, 1: (d // 2,), 3: (d // 2 - 2 * (3 * d // 16), 3 * d // 16, 3 * d // 16)}[axes]
    qw = (1 + 0.3 * torch.randn(d, generator=g)).bfloat16() if norm else None
    kw = (1 + 0.3 * torch.randn(d, generator=g)).bfloat16() if norm else None
    cache, batch = on_gpu(tlq, s)
    ws = tlq.kv_workspace(cache, heads, s["T"], batch)
    dev = qkv.cuda()
    if stride:
        dev = torch.cat([dev, torch.full((s["T"], stride), math.nan, dtype=torch.bfloat16, device="cuda")], 1)
    up = lambda v: None if v is None else v.cuda()  # noqa: E731
    q, k, v = tlq.tlq_kv_store(dev, heads, cache, batch, up(pos), up(table) if axes else None, sections, up(qw), up(kw), 1e-6,
                               want_values=True, workspace=ws)
    x = qkv.double().view(s["T"], heads + 2 * hk, d)
    want_q = ref.rotated(ref.normed(x[:, :heads], qw, 1e-6), pos, sections, table)
    want_k = ref.rotated(ref.normed(x[:, heads:heads + hk], kw, 1e-6), pos, sections, table)
    return cache, ws, q, k, v, want_q, want_k, x[:, heads + hk:]


def places(s):
    for r in range(len(s["kv"])):
        n = int(s["cu"][r + 1] - s["cu"][r])
        for i in range(n):
            p = int(s["kv"][r]) - n + i
            yield int(s["cu"][r]) + i, int(s["table"][r, p // BLOCK]), p % BLOCK


@pytest.mark.parametrize("lens", sorted(STORE_LENS))
@pytest.mark.parametrize("heads,hk,d", [(12, 2, 128), (14, 2, 64), (3, 3, 128), (8, 8, 64), (5, 1, 128)])
@pytest.mark.parametrize("norm,axes", [(True, 1), (False, 3), (True, 0)])
def test_store(tlq, heads, hk, d, lens, norm, axes):
    q_lens, kv_lens = STORE_LENS[lens]
    s = make_batch(51, q_lens, kv_lens, hk, d)
    check_store(tlq, s, heads, hk, d, norm, axes, 0)


def test_store_of_strided_rows(tlq):
    check_store(tlq, make_batch(52, [40, 3], [40, 99], 2, 128), 12, 2, 128, True, 3, 24)


def check_store(tlq, s, heads, hk, d, norm, axes, stride):
    cache, ws, q, k, v, want_q, want_k, want_v = run_store(tlq, s, heads, hk, d, norm, axes, 7, stride)
    assert tlq.tlq_read_status(ws) == tlq.OK
    # fp32 arithmetic (sum of d squares, root, two products, rotation) and one rounding to 8 bits
    size = want_q.abs().amax(-1, keepdim=True)
    assert torch.all((q.double().cpu() - want_q).abs() <= 2.0 ** -8 * want_q.abs() * (1 + 2.0 ** -7) + 2.0 ** -19 * size)
    kc, vc, ks, vs = cache.k_codes.cpu(), cache.v_codes.cpu(), cache.k_steps.cpu(), cache.v_steps.cpu()
    tops, starts = {}, {}
    for tok, blk, off in places(s):
        a, b = want_k[tok].abs().amax(1), want_v[tok].abs().amax(1)
        if blk in tops:
            tops[blk] = (torch.maximum(tops[blk][0], a), torch.maximum(tops[blk][1], b))
        else:
            tops[blk], starts[blk] = (a, b), off
    for name, steps, was, i in (("k", ks, s["ks"], 0), ("v", vs, s["vs"], 1)):
        for blk in range(len(steps)):
            if blk not in tops:
                assert torch.equal(steps[blk], was[blk]) or torch.isnan(was[blk]).all()
                continue
            want = tops[blk][i].clamp_min(ref.FLOOR) / 127
            if starts[blk] > 0:
                want = torch.maximum(want, was[blk].double())
            assert torch.all((steps[blk].double() - want).abs() <= 2.0 ** -19 * want), name
    written = torch.zeros(len(ks), BLOCK, dtype=torch.bool)
    for tok, blk, off in places(s):
        written[blk, off] = True
        for codes, step, want, val in ((kc[blk, :, off], ks[blk], want_k[tok], k[tok]), (vc[blk, :, :, off], vs[blk], want_v[tok], v[tok])):
            x = codes.float() * step[:, None]
            assert codes.abs().max() <= 127
            assert torch.all((x.double() - want).abs() <= step.double()[:, None] * (0.5 + 2.0 ** -11))
            assert torch.equal(val.cpu(), x.bfloat16())
    # older codes of the request follow the step, everything else stays
    for blk in range(len(ks)):
        old_k, old_v = s["kc"][blk].float(), s["vc"][blk].float()
        if blk in starts and starts[blk] > 0:
            for h in range(hk):
                if ks[blk, h] > s["ks"][blk, h]:
                    old_k[h, :starts[blk]] = torch.round(old_k[h, :starts[blk]] * (s["ks"][blk, h] / ks[blk, h]))
                if vs[blk, h] > s["vs"][blk, h]:
                    old_v[h, :, :starts[blk]] = torch.round(old_v[h, :, :starts[blk]] * (s["vs"][blk, h] / vs[blk, h]))
        keep = ~written[blk]
        assert torch.equal(kc[blk].float()[:, keep], old_k[:, keep])
        assert torch.equal(vc[blk].float()[:, :, keep], old_v[:, :, keep])


def test_store_twice_is_store_once(tlq):
    s = make_batch(53, [5, 70], [30, 100], 2, 128)
    cache, batch = on_gpu(tlq, s)
    qkv = torch.randn(75, 10 * 128, generator=gen(1)).bfloat16().cuda()
    tlq.tlq_kv_store(qkv, 6, cache, batch)
    first = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps)]
    tlq.tlq_kv_store(qkv, 6, cache, batch)
    for a, b in zip(first, (cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps)):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())


def test_store_token_by_token_matches_the_prompt(tlq):
    """Keys and values written one by one stay within half a step for each time the block's step grew."""
    hk, d, n = 1, 64, 100
    g = gen(9)
    qkv = torch.randn(n, 3 * d, generator=g).bfloat16().cuda()
    table = torch.tensor([[2, 0]], dtype=torch.int32).cuda()
    cache = tlq.KvCache.empty(3, hk, d, "cuda")
    grew = torch.zeros(3, hk)
    for i in range(n):
        before = cache.k_steps.cpu().clone()
        batch = tlq.KvBatch(torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([i + 1], dtype=torch.int32).cuda(), table, 1)
        tlq.tlq_kv_store(qkv[i:i + 1], 1, cache, batch)
        grew += (cache.k_steps.cpu() > before).float()
    for blk, lo, hi in ((2, 0, 64), (0, 64, 100)):
        x = cache.k_codes[blk, 0, :hi - lo].float().cpu() * cache.k_steps[blk, 0].cpu()
        want = qkv[lo:hi, d:2 * d].float().cpu()
        assert torch.all((x - want).abs() <= cache.k_steps[blk, 0].cpu() * (0.5 * grew[blk, 0] + 0.01))
        assert torch.allclose(cache.k_steps[blk, 0].cpu(), want.abs().max() / 127, rtol=1e-6)


def test_store_of_zeros_and_of_values_that_are_not_finite(tlq):
    s = make_batch(54, [10, 10], [10, 10], 1, 64)
    qkv = torch.randn(20, 3 * 64, generator=gen(2)).bfloat16()
    qkv[:10, 64:] = 0
    qkv[12, 64 + 5] = math.inf
    qkv[13, 64 + 6] = math.nan
    qkv[14, 128 + 7] = -math.inf
    cache, ws, q, k, v, *_ = run_store(tlq, s, 1, 1, 64, False, 0, 0, qkv=qkv)
    assert tlq.tlq_read_status(ws) == tlq.ERR_NONFINITE
    zero, odd = int(s["table"][0, 0]), int(s["table"][1, 0])
    assert torch.all(cache.k_codes[zero, :, :10] == 0) and torch.all(k[:10] == 0) and torch.all(v[:10] == 0)
    assert torch.allclose(cache.k_steps[zero].cpu(), torch.tensor(ref.FLOOR / 127), rtol=1e-6)
    assert int(cache.k_codes[odd, 0, 2, 5]) == 127 and int(cache.k_codes[odd, 0, 3, 6]) == 0
    assert int(cache.v_codes[odd, 0, 7, 4]) == -127
    fine = torch.isfinite(qkv[10:, 64:128].float())
    top = qkv[10:, 64:128].float()[fine].abs().max()
    assert torch.allclose(cache.k_steps[odd].cpu(), top / 127, rtol=1e-6)
    assert torch.isfinite(k.float()).all() and torch.isfinite(v.float()).all()


def test_store_reports_metadata_that_does_not_fit(tlq):
    s = make_batch(55, [1, 3], [5, 70], 1, 64)
    qkv = torch.randn(4, 4 * 64, generator=gen(2)).bfloat16().cuda()
    for what in ("block", "position", "short"):
        t = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
        pos = torch.arange(4, dtype=torch.int32)
        if what == "block":
            t["table"][0, 0] = 99
        elif what == "position":
            pos[2] = 50
        else:
            t["kv"][1] = 2                      # fewer cached tokens than new ones: the first one has no place
        cache, batch = on_gpu(tlq, t)
        ws = tlq.kv_workspace(cache, 2, 4, batch)
        q, _, _ = tlq.tlq_kv_store(qkv, 2, cache, batch, pos.cuda(), rope_table(50, 64).cuda(), workspace=ws)
        assert tlq.tlq_read_status(ws) == tlq.ERR_SHAPE
        assert torch.isfinite(q.float()).all()


# ---------------------------------------------------------------------------------------------- together

def test_store_then_attention_on_another_stream(tlq):
    """A prompt, then single tokens, written and read on a side stream, against 64 bits from what the cache holds."""
    heads, hk, d = 6, 2, 64
    g = gen(77)
    n, extra = 90, 3
    qkv = torch.randn(n + extra, (heads + 2 * hk) * d, generator=g).bfloat16().cuda()
    table = torch.tensor([[1, 3]], dtype=torch.int32).cuda()
    cache = tlq.KvCache.empty(4, hk, d, "cuda")
    ang = rope_table(200, d).cuda()
    steps = [(0, n)] + [(n + i, 1) for i in range(extra)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for at, count in steps:
            batch = tlq.KvBatch(torch.tensor([0, count], dtype=torch.int32).cuda(), torch.tensor([at + count], dtype=torch.int32).cuda(),
                                table, count)
            pos = torch.arange(at, at + count, dtype=torch.int32).cuda()
            q, _, _ = tlq.tlq_kv_store(qkv[at:at + count], heads, cache, batch, pos, ang)
            out, lse = tlq.tlq_kv_attention(q, cache, batch, d ** -0.5, want_lse=True)
            side.synchronize()
            want, wl, mag, small, weight = ref.attention(q.cpu(), cache.k_codes.cpu(), cache.v_codes.cpu(), cache.k_steps.cpu(),
                                                  cache.v_steps.cpu(), batch.cu_q.cpu(), batch.kv_len.cpu(), table.cpu(), d ** -0.5, True)
            most, most_lse = attention_bounds(want, wl, mag, small, weight, d)
            assert torch.all((out.double().cpu() - want).abs() <= most)
            assert torch.all((lse.double().cpu() - wl).abs() <= most_lse)


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 5], [300, 200]), (list(BIG[:1]) + [70], list(BIG[1:]) + [100])])
def test_blocks_beyond_four_gigabytes(tlq, q_lens, kv_lens):
    """Block numbers whose bytes lie beyond 2^32: the same bits as from a small cache."""
    hk, d, heads = 8, 128, 16
    s = make_batch(51, q_lens, kv_lens, hk, d)
    n_blocks = (1 << 32) // (hk * BLOCK * d) + s["kc"].shape[0]
    big = tlq.KvCache(*[torch.empty((n_blocks, *s[k].shape[1:]), dtype=s[k].dtype, device="cuda") for k in ("kc", "vc", "ks", "vs")])
    t = dict(s, table=s["table"] + (n_blocks - s["kc"].shape[0]))
    qkv = torch.randn(s["T"], (heads + 2 * hk) * d, generator=gen(6)).bfloat16().cuda()
    results = []
    for batch_of, cache in ((s, tlq.KvCache(*[s[k].cuda() for k in ("kc", "vc", "ks", "vs")])), (t, big)):
        for name in ("k_codes", "v_codes", "k_steps", "v_steps"):
            getattr(cache, name)[-s["kc"].shape[0]:] = s[name[:1] + name[2]].cuda()
        batch = tlq.KvBatch(s["cu"].cuda(), s["kv"].cuda(), batch_of["table"].cuda(), s["q_max"])
        ws = tlq.kv_workspace(cache, heads, s["T"], batch)
        q, _, _ = tlq.tlq_kv_store(qkv, heads, cache, batch, workspace=ws)
        out, lse = tlq.tlq_kv_attention(q, cache, batch, d ** -0.5, want_lse=True, workspace=ws)
        assert tlq.tlq_read_status(ws) == tlq.OK
        tail = [getattr(cache, name)[-s["kc"].shape[0]:].clone() for name in ("k_codes", "v_codes")]
        results.append([q, out, lse] + tail)
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_step_recorded_as_a_graph(tlq):
    """Store and attention captured once and replayed with other inputs and lengths in the same places."""
    hk, d, heads = 2, 128, 12
    s = make_batch(53, [1, 1], [150, 64], hk, d)
    lens = [s["kv"].clone(), s["kv"] - 3]
    inputs = [torch.randn(2, (heads + 2 * hk) * d, generator=gen(7 + i)).bfloat16().cuda() for i in range(2)]

    def fresh():
        return tlq.KvCache(*[s[k].cuda() for k in ("kc", "vc", "ks", "vs")])

    def step(x, cache, batch, ws):
        q, _, _ = tlq.tlq_kv_store(x, heads, cache, batch, workspace=ws)
        return tlq.tlq_kv_attention(q, cache, batch, d ** -0.5, workspace=ws)[0]

    cache, x, kv = fresh(), inputs[0].clone(), lens[0].cuda()
    batch = tlq.KvBatch(s["cu"].cuda(), kv, s["table"].cuda(), 1)
    ws = tlq.kv_workspace(cache, heads, 2, batch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, cache, batch, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step(x, cache, batch, ws)
    for i in (1, 0, 1):
        for name, k in (("k_codes", "kc"), ("v_codes", "vc"), ("k_steps", "ks"), ("v_steps", "vs")):
            getattr(cache, name).copy_(s[k])
        x.copy_(inputs[i])
        kv.copy_(lens[i])
        graph.replay()
        own = fresh()
        want = step(inputs[i], own, tlq.KvBatch(s["cu"].cuda(), lens[i].cuda(), s["table"].cuda(), 1), None)
        assert torch.equal(y, want) and torch.equal(cache.k_codes, own.k_codes) and torch.equal(cache.v_codes, own.v_codes)
        assert tlq.tlq_read_status(ws) == tlq.OK


def test_example_serves_a_calibrated_layer():
    """Prompts and answers of the example against 32-bit floats on the projections' codes.  Rounding to 8 bits is an error of
    step / sqrt(12), with the largest of some thousand values at 4 deviations 0.9 %: of the values, of attention's results, and
    of the keys, where it is multiplied by the scores' deviation (1.2 here, 2 where outliers make it so).  1.7 to 2.5 % where
    they are independent; 5 % is a wrong block."""
    import importlib.util
    import pathlib
    path = pathlib.Path(__file__).resolve().parent.parent / "examples" / "serve_layer.py"
    spec = importlib.util.spec_from_file_location("serve_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(["--requests", "3", "--prompt", "300", "--steps", "5", "--calibration", "256"]) < 0.05
