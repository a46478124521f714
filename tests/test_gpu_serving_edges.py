"""The serving operators where a step, a length or a stream is not what the ordinary case has."""
import math

import pytest
import torch

import serving_ref as ref
from test_gpu_serving import BIG, BLOCK, gen, linear_close, make_batch, on_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tlq():
    from paper_2602_07899_b200 import tlq as mod
    return mod


def test_steps_that_grow_reach_the_attention_behind_the_store(tlq):
    """Decoding steps without a pause between the calls against the same with the GPU idle between them: the kernels of one
    come up while those of the other still write the steps, codes and queries that they read."""
    hk, d, heads, n = 8, 128, 16, 24
    s = make_batch(61, [1] * 6, [40, 64, 65, 130, 200, 7], hk, d)
    s["ks"], s["vs"] = s["ks"].nan_to_num(0.0), s["vs"].nan_to_num(0.0, posinf=0.0)
    grow = torch.exp2(torch.arange(n) / 3.0)[:, None, None]        # every token is larger than those before: every step grows
    qkv = (torch.randn(n, 6, (heads + 2 * hk) * d, generator=gen(3)) * grow).bfloat16().cuda()

    def answer(pause):
        cache, batch = on_gpu(tlq, s)
        ws = tlq.kv_workspace(cache, heads, 6, batch)
        outs = []
        torch.cuda.synchronize()
        for i in range(n):
            q, _, _ = tlq.tlq_kv_store(qkv[i], heads, cache, batch, workspace=ws)
            if pause:
                torch.cuda.synchronize()
            outs.append(tlq.tlq_kv_attention(q, cache, batch, d ** -0.5 / 64, want_lse=True, workspace=ws))
            if pause:
                torch.cuda.synchronize()
        assert tlq.tlq_read_status(ws) == tlq.OK
        return [t for pair in outs for t in pair] + [cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps]

    want = answer(True)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(want, answer(False)))


def test_tensors_in_host_memory_beside_those_of_the_gpu_are_refused(tlq):
    s = make_batch(62, [1, 2], [5, 70], 1, 64)
    cache, batch = on_gpu(tlq, s)
    q, qkv = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 4 * 64, dtype=torch.bfloat16, device="cuda")
    pos, ang = torch.zeros(3, dtype=torch.int32), torch.zeros(9, 64)
    with pytest.raises(ValueError, match="device"):
        tlq.KvBatch(s["cu"], s["kv"].cuda(), s["table"].cuda(), 2)
    with pytest.raises(ValueError, match="device"):
        tlq.tlq_kv_attention(q, cache, tlq.KvBatch(s["cu"], s["kv"], s["table"], 2), 0.1)
    with pytest.raises(ValueError, match="device"):
        tlq.tlq_kv_store(qkv, 2, cache, batch, pos, ang.cuda())
    with pytest.raises(ValueError, match="device"):
        tlq.tlq_kv_store(qkv, 2, cache, batch, pos.cuda(), ang)
    x, t, w, u = torch.zeros(2, 32, dtype=torch.int8), torch.zeros(2), torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5)
    for here in (lambda v: v is not t, lambda v: v is not u, lambda v: v is not w):
        with pytest.raises(ValueError, match="device"):
            tlq.tlq_linear_i8(*[v.cuda() if here(v) else v for v in (x, t, w, u)])


@pytest.mark.parametrize("n,ci,co", [(2048, 1040, 8963), (4100, 208, 2401), (4100, 208, 2396), (700, 48, 13001)])
def test_linear_of_many_tokens_and_odd_widths(tlq, n, ci, co):
    """Widths that are no multiple of 8, and sums that end inside a block of channels, in the persistent kernel."""
    g = gen(n + ci + co)
    xq = torch.randint(-127, 128, (n, ci), generator=g).to(torch.int8).cuda()
    wq = torch.randint(-128, 128, (co, ci), generator=g).to(torch.int8).cuda()
    t, u = (torch.rand(n, generator=g) * 0.05 + 1e-4).cuda(), (torch.rand(co, generator=g) * 0.002 + 1e-6).cuda()
    b = torch.randn(co, generator=g).bfloat16().cuda()
    for bias in (b, None):
        want = (xq.double() @ wq.double().t()) * torch.outer(t.double(), u.double())     # exact: integers below 2^53
        mag = want.abs()
        if bias is not None:
            want, mag = want + bias.double(), mag + bias.double().abs()
        guarded = torch.full((n * co + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        y = tlq.tlq_linear_i8(xq, t, wq, u, bias, out=guarded[:n * co].view(n, co))
        linear_close(y, want.cpu(), mag.cpu())
        assert torch.all(guarded[n * co:] == 7.0)


@pytest.mark.parametrize("n,ci,co", [(5, 512, 96), (5, 512, 97), (60, 512, 96), (60, 512, 97), (4100, 208, 2400), (4100, 208, 2401)])
def test_linear_of_steps_that_are_not_finite(tlq, n, ci, co):
    """The same pattern of infinities and NaN whichever kernel the size selects; zero sums of an infinite step are NaN."""
    g = gen(n + co)
    xq = torch.randint(-127, 128, (n, ci), generator=g).to(torch.int8)
    wq = torch.randint(-127, 128, (co, ci), generator=g).to(torch.int8)
    t, u = torch.rand(n, generator=g) + 0.5, torch.rand(co, generator=g) + 0.5
    xq[1] = 0
    t[1], t[2], t[n - 1] = math.inf, math.inf, math.nan
    u[3], u[co - 1], u[co - 2] = math.nan, math.inf, -math.inf
    acc = xq.cuda().double() @ wq.cuda().double().t()
    want = (acc * torch.outer(t.cuda().double(), u.cuda().double())).cpu()
    y = tlq.tlq_linear_i8(xq.cuda(), t.cuda(), wq.cuda(), u.cuda()).double().cpu()
    assert torch.isnan(want).any() and torch.isinf(want).any()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    odd = torch.isinf(want)
    assert torch.equal(y[odd], want[odd])
    fine = torch.isfinite(want)
    linear_close(y[fine], want[fine], want[fine].abs())


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 2], [20000, 9]), ([300, 1], [140000, 70])])
def test_attention_over_an_empty_cache(tlq, q_lens, kv_lens):
    """Blocks that nothing was written to, as before a warm-up: all scores equal, all values zero.  The logarithm is taken of a sum
    below 2^112 (its result is exact to 2^-17), and the sums of equal powers of two are exact."""
    hk, d, heads = 1, 64, 4
    need = [-(-k // BLOCK) for k in kv_lens]
    cache = tlq.KvCache.empty(sum(need), hk, d, "cuda")
    table = torch.zeros(2, max(need), dtype=torch.int32)
    table[0, :need[0]], table[1, :need[1]] = torch.arange(need[0]), need[0] + torch.arange(need[1])
    cu = torch.tensor([0, q_lens[0], sum(q_lens)], dtype=torch.int32)
    batch = tlq.KvBatch(cu.cuda(), torch.tensor(kv_lens, dtype=torch.int32).cuda(), table.cuda(), max(q_lens))
    q = torch.randn(sum(q_lens), heads, d, generator=gen(1)).bfloat16().cuda()
    for causal in (True, False):
        out, lse = tlq.tlq_kv_attention(q, cache, batch, 0.125, causal, want_lse=True)
        assert torch.all(out == 0)
        seen = torch.cat([k - n + 1 + torch.arange(n) if causal else torch.full((n,), k) for n, k in zip(q_lens, kv_lens)])
        want = seen.double().log()[:, None].expand(-1, heads)
        assert torch.all((lse.double().cpu() - want).abs() <= 2.0 ** -15)


def dirty(*shapes):
    """Leaves NaN in the memory that the next tensors of these shapes will get."""
    held = [torch.full(shape, math.nan, dtype=dtype, device="cuda") for shape, dtype in shapes]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("big", [False, True])
@pytest.mark.parametrize("before,after", [(0, 5), (3, 0), (70, 131), (1, 1)])
def test_rows_of_no_request_are_empty_rows(tlq, before, after, big):
    """Token tensors padded at either end: attention gives zeros and -infinity there, the store zeros for keys and values."""
    hk, d, heads = 2, 128, 6
    q_lens, kv_lens = [1, 40, 0, 3] + [BIG[0]] * big, [90, 300, 64, 3] + [BIG[1]] * big
    s = make_batch(63, q_lens, kv_lens, hk, d)
    T = before + s["T"] + after
    rows = slice(before, before + s["T"])
    q = torch.randn(T, heads, d, generator=gen(4)).bfloat16().cuda()
    cache, batch = on_gpu(tlq, s)
    want, want_lse = tlq.tlq_kv_attention(q[rows], cache, batch, 0.1, want_lse=True)
    padded = tlq.KvBatch((s["cu"] + before).cuda(), batch.kv_len, batch.block_table, s["q_max"])
    ws = tlq.kv_workspace(cache, heads, T, padded)
    dirty(((T, heads, d), torch.bfloat16), ((T, heads), torch.float32))
    out, lse = tlq.tlq_kv_attention(q, cache, padded, 0.1, want_lse=True, workspace=ws)
    none = torch.ones(T, dtype=torch.bool, device="cuda")
    none[rows] = False
    assert torch.all(out[none] == 0) and torch.all(lse[none] == -math.inf)
    assert torch.equal(out[rows], want) and torch.equal(lse[rows], want_lse)
    # the store
    qkv = torch.randn(T, (heads + 2 * hk) * d, generator=gen(5)).bfloat16().cuda()
    wq, wk, wv = tlq.tlq_kv_store(qkv[rows], heads, on_gpu(tlq, s)[0], batch, want_values=True)
    cache = on_gpu(tlq, s)[0]
    dirty(((T, heads, d), torch.bfloat16), ((T, hk, d), torch.bfloat16), ((T, hk, d), torch.bfloat16))
    gq, gk, gv = tlq.tlq_kv_store(qkv, heads, cache, padded, want_values=True, workspace=ws)
    assert torch.equal(gq[rows], wq) and torch.equal(gk[rows], wk) and torch.equal(gv[rows], wv)
    assert torch.all(gk[none] == 0) and torch.all(gv[none] == 0) and torch.isfinite(gq.float()).all()
    assert tlq.tlq_read_status(ws) == tlq.OK


def test_store_values_of_tokens_without_a_place_are_zeros(tlq):
    """More new tokens than cached ones (the first have no place), a block outside of the cache, a length beyond the table."""
    hk, d, heads = 2, 64, 4
    s = make_batch(66, [5, 70, 3, 9], [2, 100, 10, 9], hk, d, pad=0)
    s["table"][1, 1] = 1 << 20
    s["kv"][3] = s["table"].shape[1] * BLOCK + 1
    gone = torch.zeros(s["T"], dtype=torch.bool, device="cuda")
    gone[:3] = True                                               # places -3 .. -1
    gone[5 + 34:5 + 70] = True                                    # places 64 .. 99 of request 1
    gone[5 + 70 + 3:] = True
    cache, batch = on_gpu(tlq, s)
    ws = tlq.kv_workspace(cache, heads, s["T"], batch)
    qkv = (torch.randn(s["T"], (heads + 2 * hk) * d, generator=gen(5)).abs() + 1).bfloat16().cuda()
    dirty(((s["T"], heads, d), torch.bfloat16), ((s["T"], hk, d), torch.bfloat16), ((s["T"], hk, d), torch.bfloat16))
    _, k, v = tlq.tlq_kv_store(qkv, heads, cache, batch, want_values=True, workspace=ws)
    assert tlq.tlq_read_status(ws) == tlq.ERR_SHAPE
    for x in (k, v):
        assert torch.all(x[gone] == 0) and torch.all(x[~gone].float().abs().amax(-1) > 0.5) and torch.isfinite(x.float()).all()


@pytest.mark.parametrize("what", ["length", "negative", "rows"])
@pytest.mark.parametrize("big", [False, True])
def test_requests_that_do_not_fit_are_left_out_whole(tlq, what, big):
    """A length beyond the table, more new tokens than the batch allows: the request's tokens have no place.  None of its
    blocks is written, its rows are empty, the other requests are unharmed."""
    hk, d, heads = 2, 64, 6
    q_lens, kv_lens = [20, 3, 40] + [BIG[0]] * big, [128, 70, 128] + [BIG[1]] * big
    s = make_batch(64, q_lens, kv_lens, hk, d, pad=0)
    if what == "length":
        s["kv"][0] = s["table"].shape[1] * BLOCK + 10
        s["table"][0] = s["table"][0, 0]
    elif what == "negative":
        s["kv"][0] = -5
    else:
        s["q_max"], out_of = (BIG[0] - 1, 3) if big else (39, 2)
    out_of = 0 if what != "rows" else out_of
    cu = [int(v) for v in s["cu"]]
    rows = torch.zeros(s["T"], dtype=torch.bool, device="cuda")
    rows[cu[out_of]:cu[out_of + 1]] = True
    qkv = torch.randn(s["T"], (heads + 2 * hk) * d, generator=gen(5)).bfloat16().cuda()
    cache, batch = on_gpu(tlq, s)
    ws = tlq.kv_workspace(cache, heads, s["T"], batch)
    q, k, _ = tlq.tlq_kv_store(qkv, heads, cache, batch, want_values=True, workspace=ws)
    assert tlq.tlq_read_status(ws) == tlq.ERR_SHAPE
    own = s["table"][out_of, :-(-kv_lens[out_of] // BLOCK)].unique().long()
    for name in ("kc", "vc", "ks", "vs"):
        got = getattr(cache, {"kc": "k_codes", "vc": "v_codes", "ks": "k_steps", "vs": "v_steps"}[name]).cpu()
        assert torch.equal(got[own], s[name][own]), name
    # the others: as without it
    fits = dict(s, kv=s["kv"].clone(), q_max=max(q_lens))
    if what != "rows":
        fits["kv"][0] = kv_lens[0]
    good, good_batch = on_gpu(tlq, fits)
    wq, wk, _ = tlq.tlq_kv_store(qkv, heads, good, good_batch, want_values=True)
    others = torch.tensor([b for b in range(len(s["ks"])) if b not in own.tolist()])
    assert torch.equal(cache.k_codes[others], good.k_codes[others]) and torch.equal(cache.v_codes[others], good.v_codes[others])
    assert torch.equal(q, wq) and torch.equal(k[~rows], wk[~rows])
    ws.zero_()
    dirty(((s["T"], heads, d), torch.bfloat16), ((s["T"], heads), torch.float32))
    out, lse = tlq.tlq_kv_attention(q, cache, batch, 0.125, want_lse=True, workspace=ws)
    assert tlq.tlq_read_status(ws) == tlq.ERR_SHAPE
    assert torch.all(out[rows] == 0) and torch.all(lse[rows] == -math.inf)
    want = ref.attention(q.cpu(), cache.k_codes.cpu(), cache.v_codes.cpu(), cache.k_steps.cpu(), cache.v_steps.cpu(), s["cu"],
                         torch.where(torch.arange(len(kv_lens)) == out_of, 0, fits["kv"]), s["table"], 0.125, True)[0]
    err = (out.double().cpu() - want).abs()
    assert torch.all(err <= 2.0 ** -6 * want.abs().amax())


def pool_of(t):
    """Stream whose pool the memory of a tensor belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]


def test_results_belong_to_the_stream_that_writes_them(tlq):
    """Memory from another stream's pool may still be in use there by what was queued before, and is given away again as soon as
    that stream's owner drops it."""
    side = torch.cuda.Stream()
    s = make_batch(65, [1, 70], [90, 100], 2, 64)
    cache, batch = on_gpu(tlq, s)
    qkv = torch.randn(s["T"], 10 * 64, generator=gen(1)).bfloat16().cuda()
    xq, wq = torch.zeros(64, 512, dtype=torch.int8, device="cuda"), torch.zeros(96, 512, dtype=torch.int8, device="cuda")
    t, u = torch.ones(64, device="cuda"), torch.ones(96, device="cuda")
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        q, k, v = tlq.tlq_kv_store(qkv, 6, cache, batch, want_values=True, stream=stream)
        out, lse = tlq.tlq_kv_attention(q, cache, batch, 0.1, want_lse=True, stream=stream)
        y = tlq.tlq_linear_i8(xq, t, wq, u, stream=stream)
        side.synchronize()
        assert [pool_of(r) for r in (q, k, v, out, lse, y)] == [side.cuda_stream] * 6
    assert pool_of(tlq.tlq_linear_i8(xq, t, wq, u)) == torch.cuda.current_stream().cuda_stream
