"""The norm with the residual's addition and an 8-bit output, and the 8-bit product with activation, gate and residual, against their
definitions in 64 bits, at the sizes and values where they can go wrong; and both as a layer uses them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tlq():
    from paper_2602_07899_b200 import tlq as mod
    return mod


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bf(t):
    return t.bfloat16().cuda()


# ---------------------------------------------------------------------------------------------- norm

def norm_ref(x, r, w, s, eps, bits):
    """(h, y, v, steps) in 64 bits; h as the residual stream holds it."""
    h = x if r is None else (x.float() + r.float()).bfloat16()
    y = h.double() / ((h.double() ** 2).mean(1, keepdim=True) + eps).sqrt()
    if w is not None:
        y = y * w.double()
    v = y if s is None else y / s.double()
    return h, y, v, v.abs().amax(1).clamp_min(1e-5) / (2 ** (bits - 1) - 1)


def check_norm(tlq, out, x, r, w, s, eps=1e-6, bits=8, what="all"):
    """The sum of squares: at most 8 + 8 + 5 + 16 additions one after another, positive terms, 2^-24 of it each; its root half of that;
    mean, rsqrt (2 units), and products of four factors 10 more: below 2^-19 of the value.  Codes: half a step more."""
    h, y, v, steps = norm_ref(x, r, w, s, eps, bits)
    assert torch.equal(out["h"].view(torch.int16), h.view(torch.int16))
    if out["y"] is not None:
        assert torch.all((out["y"].double() - y).abs() <= (2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -19) * y.abs() + 1e-40)
    if out["codes"] is not None:
        got = out["steps"].double()
        assert torch.all((got - steps).abs() <= 2.0 ** -19 * steps)
        codes = out["codes"].double()
        assert int(codes.abs().max()) <= 2 ** (bits - 1) - 1
        assert torch.all((codes * got[:, None] - v).abs() <= 0.5 * got[:, None] * (1 + 2.0 ** -15) + 2.0 ** -18 * v.abs())
    if out["values"] is not None:
        assert torch.equal(out["values"], (out["codes"].float() * out["steps"][:, None]).bfloat16())


@pytest.mark.parametrize("n", [1, 2, 3, 65, 700])
@pytest.mark.parametrize("c", [16, 128, 1536, 2048, 3584, 4112, 8192, 16400, 29568, 32768])
def test_norm_over_widths(tlq, n, c):
    g = gen(n * 31 + c)
    x, r = bf(torch.randn(n, c, generator=g) * 3), bf(torch.randn(n, c, generator=g))
    w, s = bf(1 + 0.3 * torch.randn(c, generator=g)), bf(torch.exp(torch.randn(c, generator=g)))
    for residual, weight, scales in ((r, w, s), (None, w, None), (r, None, s), (None, None, None)):
        out = tlq.tlq_norm_quantize(x, weight, residual=residual, s=scales, want_values=True, want_y=True)
        check_norm(tlq, out, x, residual, weight, scales)
    only = tlq.tlq_norm_quantize(x, w, residual=r, want_codes=False, want_y=True)
    assert only["codes"] is None and only["steps"] is None and only["values"] is None
    check_norm(tlq, only, x, r, w, None)


@pytest.mark.parametrize("bits", [2, 4, 6, 8])
def test_norm_bits_and_eps(tlq, bits):
    g = gen(bits)
    x, w = bf(torch.randn(37, 1536, generator=g) * 0.01), bf(torch.randn(1536, generator=g))
    cfg = tlq.config(tlq.W8A8_SYM, a_bits=bits)
    for eps in (1e-12, 1e-5, 0.5):
        check_norm(tlq, tlq.tlq_norm_quantize(x, w, cfg, eps=eps, want_values=True, want_y=True), x, None, w, None, eps, bits)


@pytest.mark.parametrize("n", [1, 40, 1000])
def test_norm_of_strided_rows_and_in_place(tlq, n):
    g = gen(n)
    c = 1536
    wide_x, wide_r = bf(torch.randn(n, c + 24, generator=g)), bf(torch.randn(n, 2 * c, generator=g))
    w = bf(torch.randn(c, generator=g))
    x, r = wide_x[:, 8:8 + c], wide_r[:, c:]
    check_norm(tlq, tlq.tlq_norm_quantize(x, w, residual=r, want_values=True), x, r, w, None)
    keep_x, keep_r, margin = x.clone(), r.clone(), wide_x[:, :8].clone()
    out = tlq.tlq_norm_quantize(x, w, residual=r, h=x)
    assert out["h"] is x and torch.equal(wide_x[:, :8], margin)
    check_norm(tlq, out, keep_x, keep_r, w, None)
    x.copy_(keep_x)
    out = tlq.tlq_norm_quantize(x, w, residual=r, h=r, want_y=True, want_codes=False)
    assert torch.equal(x, keep_x)
    check_norm(tlq, out, keep_x, keep_r, w, None)


def test_norm_of_rows_of_zeros_and_of_the_largest_and_smallest_numbers(tlq):
    c = 2048
    x = torch.randn(6, c, generator=gen(0))
    x[0] = 0
    x[1] *= 1e37                    # squares beyond the 32-bit range
    x[2] = 3e38
    x[3] *= 1e-30
    x[4, 1:] = 0
    x = bf(x)
    out = tlq.tlq_norm_quantize(x, None, want_values=True, want_y=True)
    check_norm(tlq, out, x, None, None, None)
    assert torch.all(out["codes"][0] == 0) and float(out["steps"][0]) == pytest.approx(1e-5 / 127, rel=1e-6)
    assert torch.isfinite(out["y"].float()).all()


def test_norm_keeps_what_is_not_finite_to_its_row(tlq):
    g = gen(1)
    x, r, w = torch.randn(300, 1536, generator=g), bf(torch.randn(300, 1536, generator=g)), bf(torch.randn(1536, generator=g))
    bad = x.clone()
    bad[0, 3], bad[7, 1535], bad[299, 0] = math.nan, math.inf, -math.inf
    clean = tlq.tlq_norm_quantize(bf(x), w, residual=r, want_values=True, want_y=True)
    out = tlq.tlq_norm_quantize(bf(bad), w, residual=r, want_values=True, want_y=True)
    hit = torch.zeros(300, dtype=torch.bool, device="cuda")
    hit[[0, 7, 299]] = True
    for name in ("codes", "steps", "values", "y"):
        assert torch.equal(out[name][~hit], clean[name][~hit])
    assert torch.all(out["codes"][hit] == 0)
    for name in ("steps", "values", "y"):
        assert torch.isnan(out[name][hit].float()).all()
    # a product of such a row is not a number, and of the others what it was
    wq, u = torch.ones(8, 1536, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    y = tlq.tlq_linear_i8(out["codes"], out["steps"], wq, u)
    assert torch.isnan(y[hit].float()).all() and torch.isfinite(y[~hit].float()).all()


def test_norm_repeats_bit_for_bit_on_another_stream_and_in_a_graph(tlq):
    g = gen(2)
    x, r, w = bf(torch.randn(500, 3584, generator=g)), bf(torch.randn(500, 3584, generator=g)), bf(torch.randn(3584, generator=g))
    a = tlq.tlq_norm_quantize(x, w, residual=r, want_values=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = tlq.tlq_norm_quantize(x, w, residual=r, want_values=True, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = tlq.tlq_norm_quantize(x, w, residual=r, want_values=True)
    for v in c.values():
        if v is not None:
            v.zero_()
    graph.replay()
    for name in ("h", "codes", "steps", "values"):
        assert torch.equal(a[name], b[name]) and torch.equal(a[name], c[name])


def test_norm_of_no_rows(tlq):
    out = tlq.tlq_norm_quantize(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), None)
    assert out["codes"].shape == (0, 64) and out["steps"].shape == (0,)
    x, w = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = tlq.tlq_norm_quantize(x, w, residual=x, s=w, want_values=True, want_y=True)
    assert out["values"].shape == out["y"].shape == out["h"].shape == (0, 64)


def test_norm_is_what_the_activation_quantizer_makes_of_the_same_values(tlq):
    """From y in 16 bits the quantizer gives the same codes but where its rounding of y moves one across a border: one level at most."""
    g = gen(3)
    x, w, s = bf(torch.randn(64, 3584, generator=g)), bf(torch.randn(3584, generator=g)), bf(torch.rand(3584, generator=g) + 0.5)
    out = tlq.tlq_norm_quantize(x, w, s=s, want_y=True)
    codes, steps = tlq.tlq_quantize_activations(out["y"], s, tlq.config(tlq.W8A8_SYM))
    assert torch.all((steps - out["steps"]).abs() <= 2.0 ** -7 * steps)
    assert int((codes.int() - out["codes"].int()).abs().max()) <= 1


# ---------------------------------------------------------------------------------------------- product

def product_case(n, ci, co, seed=0):
    g = gen(seed + n * 7 + ci * 3 + co)
    xq = torch.randint(-127, 128, (n, ci), generator=g).to(torch.int8).cuda()
    wq = torch.randint(-128, 128, (co, ci), generator=g).to(torch.int8).cuda()
    t = (torch.rand(n, generator=g) * 0.05 + 1e-3).cuda()
    u = ((torch.rand(co, generator=g) + 0.1) * 0.01 * ci ** -0.5).cuda()
    return xq, t, wq, u, bf(torch.randn(co, generator=g))


def activate(z, act):
    if act == 1:
        return z * torch.sigmoid(z)
    if act == 2:
        return z * torch.special.ndtr(z)
    if act == 3:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def product_ref(xq, t, wq, u, b, act, gated, res):
    """(result, what its error may be before the rounding) in 64 bits.  z: four roundings to fp32 of terms of magnitude mag, 2^-21 mag.
    Slopes of the activations are below 1.2.  The activation's own error: (|z| + 8) 2^-22 of its value from the exponential's argument
    (GELU: z^2 2^-23), below 2^-14.5 of it for |z| < 200, and 1e-35 where its denominator leaves the 32-bit range; GELU's tail is a fit
    within 2^-13.4 of it, and the result is the tail times z, or z less that, which is as large at least: together below 2^-12.7."""
    acc = xq.double() @ wq.double().t()
    z = acc * torch.outer(t.double(), u.double())
    mag = z.abs()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    dz = 2.0 ** -21 * mag
    if gated:
        a, up = activate(z[:, ::2], act), z[:, 1::2]
        y, dy = a * up, (1.2 * dz[:, ::2] + 2.0 ** -12.7 * a.abs() + 1e-35) * up.abs() + a.abs() * dz[:, 1::2]
    else:
        y = activate(z, act)
        dy = 1.2 * dz + 2.0 ** -12.7 * y.abs() * (act != 0) + 1e-35
    if res is not None:
        y, dy = y + res.double(), dy + 2.0 ** -23 * (y.abs() + res.double().abs())
    return y, dy


def product_close(y, want, dy):
    assert torch.all((y.double() - want).abs() <= 2.0 ** -8 * (want.abs() + dy) + dy * 1.01 + 2.0 ** -134)


SHAPES = [(1, 16, 2), (3, 48, 18), (8, 208, 130), (9, 1040, 264), (16, 3584, 512), (17, 3584, 512), (33, 208, 30), (100, 1040, 514), (129, 3584, 520),
          (257, 208, 1030), (515, 1040, 264), (1031, 1280, 5120), (2100, 512, 4100), (2100, 512, 4108), (2100, 512, 4102), (1, 3584, 18944), (40, 8960, 1536), (300, 144, 40000)]


@pytest.mark.parametrize("n,ci,co", SHAPES)
def test_product_with_activation_gate_and_residual(tlq, n, ci, co):
    xq, t, wq, u, b = product_case(n, ci, co)
    g = gen(5)
    for act in range(4):
        for gated in (False, True):
            width = co // 2 if gated else co
            bias = b if (act + gated) % 2 else None
            wide = bf(torch.randn(n, width + 3, generator=g))
            for res in (None, wide[:, :width].contiguous(), wide[:, 1:1 + width]):
                want, dy = product_ref(xq, t, wq, u, bias, act, gated, res)
                product_close(tlq.tlq_linear_i8_act(xq, t, wq, u, bias, act, gated, res), want, dy)


@pytest.mark.parametrize("n,co", [(1, 17), (20, 17), (200, 515), (2100, 4101), (1, 5119)])
def test_product_of_odd_widths(tlq, n, co):
    xq, t, wq, u, b = product_case(n, 512, co)
    res = bf(torch.randn(n, co, generator=gen(1)))
    want, dy = product_ref(xq, t, wq, u, b, 1, False, res)
    product_close(tlq.tlq_linear_i8_act(xq, t, wq, u, b, 1, False, res), want, dy)


@pytest.mark.parametrize("n,ci,co", [(1, 512, 96), (16, 3584, 512), (40, 3584, 514), (129, 1040, 257), (2100, 512, 4100), (2100, 512, 4104)])
def test_product_without_an_epilogue_is_the_plain_product(tlq, n, ci, co):
    """Bit for bit without a bias.  With one, a product and its addition may be rounded as one where the plain call rounds both, which is 2^-24
    of the terms: the roundings to bf16 of two numbers that near are the same or next to each other."""
    xq, t, wq, u, b = product_case(n, ci, co)
    assert torch.equal(tlq.tlq_linear_i8_act(xq, t, wq, u), tlq.tlq_linear_i8(xq, t, wq, u))
    a, p = tlq.tlq_linear_i8_act(xq, t, wq, u, b).float(), tlq.tlq_linear_i8(xq, t, wq, u, b).float()
    _, dy = product_ref(xq, t, wq, u, b, 0, False, None)
    assert torch.all((a - p).abs() <= 2.0 ** -7 * p.abs() + dy)


@pytest.mark.parametrize("n,co", [(2, 96), (24, 640), (150, 515), (2100, 4096), (2100, 4101)])
def test_product_adds_to_the_residual_in_place(tlq, n, co):
    xq, t, wq, u, _ = product_case(n, 512, co)
    stream = bf(torch.randn(n, co, generator=gen(2)))
    want = tlq.tlq_linear_i8_act(xq, t, wq, u, residual=stream)
    out = tlq.tlq_linear_i8_act(xq, t, wq, u, residual=stream, out=stream)
    assert out is stream and torch.equal(out, want)


@pytest.mark.parametrize("n", [1, 30, 300, 2100])
def test_product_of_large_sums_stays_where_the_activation_sends_it(tlq, n):
    """Far to the left an activation is a (negative) zero, far to the right its argument; sums that are not finite stay so."""
    ci, co = 256, 4096 if n > 1000 else 64
    xq = torch.full((n, ci), 100, dtype=torch.int8, device="cuda")
    wq = torch.full((co, ci), 100, dtype=torch.int8, device="cuda")
    wq[1::2] = -100
    t, u = torch.ones(n, device="cuda"), torch.full((co,), 1e-3, device="cuda")
    for act in (1, 2, 3):
        y = tlq.tlq_linear_i8_act(xq, t, wq, u, act=act).float()
        assert torch.all(y[:, ::2] == torch.tensor(2560.0).bfloat16().float().item()) and torch.all(y[:, 1::2] == 0)
    t[0] = math.nan
    y = tlq.tlq_linear_i8_act(xq, t, wq, u, act=1, gated=True)
    assert torch.isnan(y[0].float()).all() and torch.isfinite(y[1:].float()).all()


def test_product_repeats_bit_for_bit_on_another_stream_and_in_a_graph(tlq):
    for n, co in ((4, 512), (24, 512), (150, 512), (2100, 4096)):
        xq, t, wq, u, b = product_case(n, 1024, co)
        ws = tlq.linear_workspace(n, 1024, co, "cuda")
        y = tlq.tlq_linear_i8_act(xq, t, wq, u, b, 1, True, workspace=ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        z = tlq.tlq_linear_i8_act(xq, t, wq, u, b, 1, True, workspace=ws, stream=side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c = tlq.tlq_linear_i8_act(xq, t, wq, u, b, 1, True, workspace=ws)
        c.zero_()
        graph.replay()
        assert torch.equal(y, z) and torch.equal(y, c) and tlq.tlq_read_status(ws) == tlq.OK


def test_product_of_no_tokens(tlq):
    xq, t, wq, u, b = product_case(0, 64, 32)
    assert tlq.tlq_linear_i8_act(xq, t, wq, u, b, 1, True).shape == (0, 16)


# ---------------------------------------------------------------------------------------------- a layer's second half

@pytest.mark.parametrize("n", [1, 19, 300])
def test_norm_gate_down_and_residual_in_a_row(tlq, n):
    """attention's output + stream -> norm -> gated product -> quantizer -> down product + stream, against the same in 64 bits on the values
    that each call's codes stand for."""
    g = gen(n)
    c, inner = 1536, 2240
    x, r, w = bf(torch.randn(n, c, generator=g)), bf(torch.randn(n, c, generator=g)), bf(1 + 0.2 * torch.randn(c, generator=g))
    s1, s2 = bf(torch.rand(c, generator=g) + 0.5), bf(torch.rand(inner, generator=g) + 0.5)
    cfg = tlq.config(tlq.W8A8_SYM)
    gate, up, down = (bf(torch.randn(o, i, generator=g) * i ** -0.5) for o, i in ((inner, c), (inner, c), (c, inner)))
    kept = [tlq.tlq_quantize_weights(m, s, cfg) for m, s in ((gate, s1), (up, s1), (down, s2))]
    wq, u = tlq.gated_rows(kept[0]["codes"], kept[1]["codes"]), tlq.gated_rows(kept[0]["steps"], kept[1]["steps"])
    first = tlq.tlq_norm_quantize(x, w, cfg, residual=r, s=s1)
    mid = tlq.tlq_linear_i8_act(first["codes"], first["steps"], wq, u, act=tlq.ACT_SILU, gated=True)
    codes, steps = tlq.tlq_quantize_activations(mid, s2, cfg)
    out = tlq.tlq_linear_i8_act(codes, steps, kept[2]["codes"], kept[2]["steps"], residual=first["h"])
    check_norm(tlq, first, x, r, w, s1)
    product_close(mid, *product_ref(first["codes"], first["steps"], wq, u, None, 1, True, None))
    product_close(out, *product_ref(codes, steps, kept[2]["codes"], kept[2]["steps"], None, 0, False, first["h"]))
    # the same block without quantized activations and weights: rounding to 8 bits only.  A step is amax / 127, its error a step / sqrt 12,
    # relative to the values amax / rms / 440: 8 / 440 = 1.8 % for a normal sample over s and for a row of weights times s, together 2.6 % of
    # each projection, times 1.2 sqrt 2 for the gated product 4.4 %; its values are products (amax / rms to 25: 5.7 %), the last weights
    # 1.8 %: root of the squares 7.4 %
    h = (x.float() + r.float()).bfloat16().double()
    y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * w.double()
    m = activate(y @ gate.double().t(), 1) * (y @ up.double().t())
    assert float((out.double() - h - m @ down.double().t()).norm() / (m @ down.double().t()).norm()) < 0.075


@pytest.mark.parametrize("c", [128, 3584])
@pytest.mark.parametrize("bits", [2, 8])
def test_norm_of_steps_near_the_end_of_the_range(tlq, c, bits):
    g = gen(c)
    x, w = torch.randn(5, c, generator=g).clamp(-2, 2), torch.full((c,), 2.0 ** 126)
    x[:, 7] = 2.0
    x, w = bf(x), bf(w)
    out = tlq.tlq_norm_quantize(x, w, tlq.config(tlq.W8A8_SYM, a_bits=bits), want_values=True)
    check_norm(tlq, out, x, None, w, None, bits=bits)
    assert int(out["codes"].abs().max()) == 2 ** (bits - 1) - 1
