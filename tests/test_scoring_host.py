"""Refusals of the norm, the product with an epilogue and the scoring calls, all on the host: no call here reaches a GPU."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry

I8, I32, F32, BF16 = torch.int8, torch.int32, torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def tlq():
    entry.build()
    from paper_2602_07899_b200 import tlq as mod
    return mod


@pytest.fixture(scope="module")
def addr():
    buf = (ctypes.c_uint8 * (1 << 20))()
    addr.keep = buf
    return (ctypes.addressof(buf) + 255) // 256 * 256


def no_device(tlq, call):
    if not torch.cuda.is_available():
        assert call() == tlq.ERR_CUDA


def test_norm_refusals(tlq, addr):
    a, good = addr, tlq.config(tlq.W8A8_SYM)

    def call(x=a, n=4, c=64, ldx=64, r=None, ldr=0, w=None, eps=1e-6, s=None, cfg=good, h=None, ldh=0, codes=a + 4096, steps=a + 8192, values=None,
             y=None):
        return tlq.lib.tlq_norm_quantize(x, n, c, ldx, r, ldr, w, eps, s, None if cfg is None else ctypes.byref(cfg), h, ldh, codes, steps, values, y,
                                         None)

    for bad in (dict(n=-1), dict(c=0), dict(c=24), dict(c=8), dict(c=32784), dict(ldx=56), dict(ldx=68), dict(r=a + 512, ldr=32), dict(r=a, ldr=65),
                dict(h=a + 512, ldh=8), dict(h=a, ldh=66), dict(n=1 << 31), dict(ldx=1 << 41)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    only_y = dict(codes=None, steps=None, y=a + 4096)
    for bad in (dict(x=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(steps=None), dict(cfg=None), dict(codes=None),
                dict(codes=None, steps=None), dict(only_y, s=a), dict(only_y, values=a + 16384), dict(only_y, steps=a + 8192),
                dict(cfg=tlq.Config(8, 1, 8, 8, 0, 1, 0, 0))):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(cfg=tlq.config()), dict(cfg=tlq.config(tlq.W8A8_SYM, a_bits=9)), dict(cfg=tlq.config(tlq.W8A8_SYM, a_bits=1))):
        assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
    for bad in (dict(x=a + 8), dict(r=a + 2, ldr=64), dict(w=a + 4), dict(s=a + 8), dict(h=a + 8, ldh=64), dict(codes=a + 8), dict(values=a + 2), dict(y=a + 4)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    # outputs over inputs or over one another, but the sum over what it is the sum of
    for bad in (dict(codes=a), dict(values=a + 256), dict(y=a + 4096), dict(h=a + 128, ldh=64), dict(h=a, ldh=72), dict(s=a + 4096), dict(steps=a + 4100),
                dict(w=a + 8192), dict(h=a + 4096, ldh=64)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for fine in (dict(), only_y, dict(h=a, ldh=64), dict(r=a + 1024, ldr=64, h=a + 1024, ldh=64), dict(r=a, ldr=64), dict(w=a + 600 * 16, s=a + 600 * 16),
                 dict(only_y, cfg=None), dict(cfg=tlq.config(tlq.W8A8_SYM, a_bits=2))):
        no_device(tlq, lambda: call(**fine))


def test_product_refusals(tlq, addr):
    a = addr

    def call(x=a, t=a, n=4, ci=64, w=a, u=a, co=8, bias=None, act=1, gated=0, res=None, ldr=0, ws=a, size=1 << 30, y=a + 4096):
        return tlq.lib.tlq_linear_i8_act(x, t, n, ci, w, u, co, bias, act, gated, res, ldr, ws, size, y, None)

    for bad in (dict(ci=0), dict(ci=72), dict(ci=131072), dict(co=0), dict(n=-1), dict(co=7, gated=1), dict(res=a, ldr=7), dict(res=a, ldr=-8),
                dict(gated=1, res=a, ldr=3)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(x=None), dict(t=None), dict(w=None), dict(u=None), dict(y=None), dict(ws=None), dict(act=-1), dict(act=4),
                dict(res=a + 4096, ldr=16), dict(res=a + 4098, ldr=8), dict(res=a + 4096 - 16, ldr=8)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(x=a + 8), dict(w=a + 4), dict(y=a + 2), dict(ws=a + 8)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    assert call(size=16) == tlq.ERR_WORKSPACE
    for fine in (dict(), dict(res=a + 4096, ldr=8), dict(res=a + 2, ldr=9), dict(gated=1, res=a + 4096, ldr=4)):
        no_device(tlq, lambda: call(**fine))


def test_logprobs_refusals(tlq, addr):
    a, o = addr, addr + 8192

    def call(z=a, dt=0, n=4, v=100, ld=100, scale=1.0, ids=None, k=0, logp=None, ent=None, lse=o, tid=None, tlp=None):
        return tlq.lib.tlq_token_logprobs(z, dt, n, v, ld, scale, ids, k, logp, ent, lse, tid, tlp, None)

    for bad in (dict(n=-1), dict(v=0), dict(v=(1 << 24) + 1, ld=1 << 25), dict(ld=99), dict(ld=0), dict(ld=1 << 33), dict(k=-1), dict(k=129, tid=o, tlp=o),
                dict(n=1 << 28)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(z=None), dict(dt=2), dict(dt=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(scale=2.0 ** 17),
                dict(scale=2.0 ** -17), dict(lse=None), dict(ids=a), dict(logp=a), dict(k=3), dict(k=3, tid=o), dict(tid=o, tlp=o), dict(lse=a), dict(lse=a + 700),
                dict(ids=o, logp=o + 8), dict(k=3, tid=a + 8, tlp=o + 4096), dict(ent=o), dict(ent=o + 12), dict(k=3, tid=o + 4096, tlp=o + 4140),
                dict(k=3, tid=o + 8, tlp=o + 4096)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(z=a + 1), dict(z=a + 2, dt=1)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    for fine in (dict(), dict(z=a + 2), dict(z=a + 4, dt=1), dict(k=128, tid=o + 4096, tlp=o + 8192), dict(ids=a, logp=o, lse=None), dict(scale=2.0 ** -16), dict(scale=2.0 ** 16)):
        no_device(tlq, lambda: call(**fine))


def test_distill_refusals(tlq, addr):
    a = addr

    def call(z=a, dt=0, n=4, v=100, ld=100, scale=1.0, ids=a + 8192, top=a + 8192, k=5, w=None, loss=a + 12288, grad=None, ldg=0):
        return tlq.lib.tlq_distill_loss(z, dt, n, v, ld, scale, ids, top, k, w, loss, grad, ldg, None)

    for bad in (dict(n=-1), dict(v=0), dict(ld=99), dict(k=0), dict(k=129), dict(grad=a + 4096, ldg=99), dict(grad=a + 4096, ldg=0)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(z=None), dict(dt=3), dict(scale=0.0), dict(scale=NAN), dict(ids=None), dict(top=None), dict(loss=None), dict(grad=a + 2, ldg=100),
                dict(grad=a, ldg=104), dict(grad=a + 200, ldg=100), dict(grad=a + 8192, ldg=100), dict(grad=a + 12288, ldg=100),
                dict(grad=a + 4096, ldg=100, w=a + 4200), dict(loss=a), dict(loss=a + 8192), dict(w=a + 12288)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(z=a + 1), dict(grad=a + 4097, ldg=100), dict(dt=1, grad=a + 4098, ldg=100)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    for fine in (dict(), dict(grad=a, ldg=100), dict(grad=a + 4096, ldg=101), dict(w=a)):
        no_device(tlq, lambda: call(**fine))


@pytest.fixture
def host():
    """Arguments that are right in everything but that they lie in host memory."""
    x = torch.zeros(2, 32, dtype=BF16)
    return dict(norm=dict(x=x, w=None), product=dict(Xq=torch.zeros(2, 32, dtype=I8), t=torch.zeros(2), Wq=torch.zeros(8, 32, dtype=I8), u=torch.zeros(8)),
                logprobs=dict(logits=x, want_lse=True),
                distill=dict(logits=x, top_ids=torch.zeros(2, 3, dtype=I32), top_logits=torch.zeros(2, 3)))


def calls(tlq):
    return dict(norm=tlq.tlq_norm_quantize, product=tlq.tlq_linear_i8_act, logprobs=tlq.tlq_token_logprobs, distill=tlq.tlq_distill_loss)


@pytest.mark.parametrize("name", ["norm", "product", "logprobs", "distill"])
def test_tensors_in_host_memory_are_refused(tlq, host, name):
    with pytest.raises(ValueError, match="device"):
        calls(tlq)[name](**host[name])


def test_binding_refuses_wrong_types_and_layouts(tlq, host):
    x = host["norm"]["x"]
    wrong = {
        "norm": (dict(x=x.float()), dict(x=x.t()), dict(residual=x[:1]), dict(residual=x.half()), dict(w=torch.zeros(31, dtype=BF16)),
                 dict(w=torch.zeros(32)), dict(s=torch.zeros(64, dtype=BF16)[::2]), dict(want_codes=False, want_values=True), dict(h=x[:1]), dict(residual=x[0]), dict(h=x[0]),
                 dict(want_codes=False, want_y=True, s=x[0]), dict(h=x.float())),
        "product": (dict(Xq=x), dict(t=torch.zeros(3)), dict(u=torch.zeros(7)), dict(Wq=torch.zeros(8, 16, dtype=I8)), dict(bias=torch.zeros(8)),
                    dict(residual=torch.zeros(2, 8)), dict(residual=torch.zeros(8, dtype=BF16)), dict(residual=torch.zeros(2, 4, dtype=BF16)), dict(gated=True, residual=torch.zeros(2, 8, dtype=BF16)),
                    dict(residual=torch.zeros(2, 16, dtype=BF16)[:, ::2]), dict(workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 12))),
        "logprobs": (dict(logits=x.half()), dict(logits=x[0]), dict(logits=x.t()), dict(ids=torch.zeros(2)), dict(ids=torch.zeros(3, dtype=I32)),
                     dict(ids=torch.zeros(4, dtype=I32)[::2]), dict(top_k=129), dict(top_k=-1)),
        "distill": (dict(logits=x.half()), dict(top_ids=torch.zeros(2, 3)), dict(top_ids=torch.zeros(3, 3, dtype=I32)), dict(top_logits=torch.zeros(2, 4)),
                    dict(top_logits=torch.zeros(2, 3).half()), dict(weights=torch.zeros(3)), dict(weights=torch.zeros(2).double())),
    }
    for name, cases in wrong.items():
        for bad in cases:
            with pytest.raises(ValueError):
                calls(tlq)[name](**{**host[name], **bad})


def test_rows_of_gate_and_up_alternate(tlq):
    gate, up = torch.arange(6, dtype=I8).view(3, 2), -torch.arange(6, dtype=I8).view(3, 2)
    both = tlq.gated_rows(gate, up)
    assert both.is_contiguous() and torch.equal(both[::2], gate) and torch.equal(both[1::2], up)
    assert torch.equal(tlq.gated_rows(gate[:, 0], up[:, 0])[::2], gate[:, 0])
    for bad in ((gate, up[:2]), (gate, up.float())):
        with pytest.raises(ValueError):
            tlq.gated_rows(*bad)
