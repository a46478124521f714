"""Refusals of the serving calls, all on the host: no call here reaches a GPU."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def tlq():
    entry.build()
    from paper_2602_07899_b200 import tlq as mod
    return mod


@pytest.fixture(scope="module")
def addr():
    buf = (ctypes.c_uint8 * 8192)()
    addr.keep = buf
    return (ctypes.addressof(buf) + 255) // 256 * 256


def structs(tlq, a, **over):
    c = dict(struct_size=ctypes.sizeof(tlq._KvCacheStruct), n_kv_heads=2, head_dim=64, n_blocks=4, k_codes=a, v_codes=a, k_steps=a, v_steps=a)
    b = dict(struct_size=ctypes.sizeof(tlq._KvBatchStruct), n_requests=2, max_q_len=4, max_blocks=3, cu_q=a, kv_len=a, block_table=a)
    for k, v in over.items():
        (c if k in c and not k.startswith("b_") else b)[k[2:] if k.startswith("b_") else k] = v
    return tlq._KvCacheStruct(**c), tlq._KvBatchStruct(**b)


def test_struct_layouts(tlq):
    assert ctypes.sizeof(tlq._KvCacheStruct) == 48 and ctypes.sizeof(tlq._KvBatchStruct) == 40


def test_linear_refusals(tlq, addr):
    L, a = tlq.lib, addr

    def call(x=a, t=a, n=4, ci=64, w=a, u=a, co=8, bias=None, ws=a, size=1 << 30, y=a):
        return L.tlq_linear_i8(x, t, n, ci, w, u, co, bias, ws, size, y, None)

    for bad in (dict(ci=0), dict(ci=72), dict(ci=131072), dict(co=0), dict(n=-1)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(x=None), dict(t=None), dict(w=None), dict(u=None), dict(y=None), dict(ws=None)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(x=a + 8), dict(w=a + 4), dict(y=a + 2), dict(ws=a + 8)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    assert call(size=16) == tlq.ERR_WORKSPACE
    assert L.tlq_linear_i8_workspace_bytes(4, 72, 8) == 0 and L.tlq_linear_i8_workspace_bytes(0, 64, 8) >= 256
    if not torch.cuda.is_available():
        assert call() == tlq.ERR_CUDA


def test_store_refusals(tlq, addr):
    L, a = tlq.lib, addr

    def call(qkv=a, T=4, ld=8 * 64, heads=4, pos=a, axes=1, sec=None, cs=a, limit=10, qw=None, kw=None, eps=1e-6, q=a, kv=None, vv=None,
             ws=a, size=1 << 30, **over):
        c, b = structs(tlq, a, **over)
        s = None if sec is None else (ctypes.c_int32 * len(sec))(*sec)
        return L.tlq_kv_store(qkv, T, ld, heads, c, b, pos, axes, s, cs, limit, qw, kw, eps, q, kv, vv, ws, size, None)

    for bad in (dict(T=-1), dict(ld=8 * 64 - 8), dict(ld=8 * 64 + 4), dict(heads=3), dict(heads=0), dict(n_kv_heads=0), dict(n_blocks=0),
                dict(n_requests=0), dict(n_requests=70000), dict(max_q_len=-1), dict(max_blocks=0), dict(limit=0),
                dict(axes=3, sec=(16, 8, 9)), dict(axes=3, sec=(16, 8, 7)), dict(axes=3, sec=(40, -4, -4)), dict(sec=(31,))):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(qkv=None), dict(q=None), dict(ws=None), dict(cs=None), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(axes=3), dict(k_codes=None), dict(v_steps=None), dict(cu_q=None), dict(block_table=None), dict(struct_size=8),
                dict(b_struct_size=8)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(head_dim=96), dict(axes=2)):
        assert call(**bad) == tlq.ERR_UNSUPPORTED, bad
    for bad in (dict(qkv=a + 8), dict(q=a + 2), dict(kv=a + 4), dict(qw=a + 2), dict(k_codes=a + 8), dict(cs=a + 4)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    assert call(size=1000) == tlq.ERR_WORKSPACE
    if not torch.cuda.is_available():
        assert call() == tlq.ERR_CUDA
        assert call(pos=None, cs=None, axes=0, limit=0) == tlq.ERR_CUDA       # nothing to rotate: not looked at


def test_attention_refusals(tlq, addr):
    L, a = tlq.lib, addr

    def call(q=a, T=4, ld=4 * 64, heads=4, scale=0.1, causal=1, ws=a, size=1 << 30, out=a, lse=None, **over):
        c, b = structs(tlq, a, **over)
        return L.tlq_kv_attention(q, T, ld, heads, c, b, scale, causal, ws, size, out, lse, None)

    for bad in (dict(T=-1), dict(ld=4 * 64 - 8), dict(ld=4 * 64 + 4), dict(heads=5), dict(n_blocks=0), dict(n_requests=0)):
        assert call(**bad) == tlq.ERR_SHAPE, bad
    for bad in (dict(q=None), dict(out=None), dict(ws=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(kv_len=None), dict(k_steps=None), dict(struct_size=0)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    for bad in (dict(q=a + 8), dict(out=a + 8), dict(ws=a + 4), dict(v_codes=a + 8)):
        assert call(**bad) == tlq.ERR_ALIGN, bad
    assert call(head_dim=32) == tlq.ERR_UNSUPPORTED
    assert call(size=1000) == tlq.ERR_WORKSPACE
    c, b = structs(tlq, a, head_dim=96)
    assert L.tlq_kv_workspace_bytes(c, b, 4, 4) == 0
    if not torch.cuda.is_available():
        assert call() == tlq.ERR_CUDA


def test_binding_refuses_wrong_types_and_layouts(tlq):
    i8, f32, bf = torch.int8, torch.float32, torch.bfloat16
    x, t, w, u = torch.zeros(2, 32, dtype=i8), torch.zeros(2), torch.zeros(5, 32, dtype=i8), torch.zeros(5)
    for bad in ((x.float(), t, w, u), (x, t.double(), w, u), (x, t[:1], w, u), (x, t, w[:, :16], u), (x, t, w, u[:3]),
                (x[:, ::2], t, w[:, ::2], u)):
        with pytest.raises(ValueError):
            tlq.tlq_linear_i8(*bad)
    kc, st = torch.zeros(3, 2, 64, 64, dtype=i8), torch.zeros(3, 2, dtype=f32)
    cache = tlq.KvCache(kc, kc.clone(), st, st.clone())
    for bad in ((kc.float(), kc, st, st), (kc, kc[:2], st, st), (kc, kc, st[:, :1], st), (kc[:, :, :32], kc, st, st),
                (kc.transpose(0, 1), kc, st, st)):
        with pytest.raises(ValueError):
            tlq.KvCache(*bad)
    i32 = torch.int32
    cu, kv, tab = torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(2, 4, dtype=i32)
    batch = tlq.KvBatch(cu, kv, tab, 1)
    for bad in ((cu[:2], kv, tab), (cu, kv.long(), tab), (cu, kv, tab[:1]), (cu, kv, tab[:, ::2])):
        with pytest.raises(ValueError):
            tlq.KvBatch(*bad, 1)
    q = torch.zeros(2, 4, 64, dtype=bf)
    for bad in (q.float(), torch.zeros(2, 4, 128, dtype=bf), torch.zeros(2, 4, 128, dtype=bf)[..., ::2], torch.zeros(2, 8, 64, dtype=bf)[:, ::2]):
        with pytest.raises(ValueError):
            tlq.tlq_kv_attention(bad, cache, batch, 0.1)
    qkv = torch.zeros(2, 8 * 64, dtype=bf)
    for bad in (dict(qkv=qkv[:, :-64]), dict(qkv=qkv.float()), dict(positions=torch.zeros(2, dtype=i32)),
                dict(positions=torch.zeros(3, dtype=i32), cos_sin=torch.zeros(4, 64)),
                dict(positions=torch.zeros(2, dtype=i32), cos_sin=torch.zeros(4, 32)), dict(q_norm=torch.zeros(32, dtype=bf)),
                dict(k_norm=torch.zeros(64))):
        with pytest.raises(ValueError):
            tlq.tlq_kv_store(**{"qkv": qkv, "n_heads": 4, "cache": cache, "batch": batch, **bad})
