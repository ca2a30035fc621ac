"""Refusals and sizes of the decoder's operators: argument errors come back before anything is launched (no GPU)."""
import pytest

from paper_1911_08076_gb300 import ifq

FAKE = 1 << 20     # never dereferenced
E = ifq


def _status(f, *a, **k):
    with pytest.raises(ifq.IfqError) as e:
        f(*a, **k)
    return e.value.status


def test_cache_sizes():
    assert ifq.ifq_kv4_cache_bytes(ifq.kv4_cache(3, 64, 8, 128)) == 3 * 8 * 4 * (16 * 128 + 128)
    assert ifq.ifq_kv4_cache_bytes(ifq.kv4_cache(1, 16, 1, 64)) == 1152
    assert ifq.ifq_kv4_cache_bytes(ifq.kv4_cache(1 << 20, 128, 8, 256)) == (1 << 20) * 8 * 8 * 4224
    for c, s in ((ifq.kv4_cache(0, 16, 1, 64), E.IFQ_EINVAL), (ifq.kv4_cache(1, 0, 1, 64), E.IFQ_EINVAL),
                 (ifq.kv4_cache(1, 24, 1, 64), E.IFQ_ESHAPE), (ifq.kv4_cache(1, 16, 0, 64), E.IFQ_EINVAL),
                 (ifq.kv4_cache(1, 16, 1, 96), E.IFQ_EUNSUPPORTED), (ifq.kv4_cache(1, 16, -1, 64), E.IFQ_EINVAL),
                 (ifq.kv4_cache(2 ** 31 - 1, 2 ** 31 - 16, 65536, 256), E.IFQ_ERANGE)):
        assert _status(ifq.ifq_kv4_cache_bytes, c) == s


def _append(status, q=FAKE, k=FAKE, v=FAKE, cos=FAKE, sin=FAKE, pos=FAKE, slots=FAKE, q_out=FAKE, cache=FAKE,
            pool=None, **kw):
    a = dict(tokens=4, q_heads=8, dtype=ifq.IFQ_BF16, rope=ifq.IFQ_ROPE_HALVES, rot_dim=128, positions=10)
    a.update(kw)
    d = ifq.kv4_append_desc(pool or ifq.kv4_cache(2, 16, 2, 128), **a)
    assert _status(ifq.ifq_kv4_append, d, q, k, v, cos, sin, pos, slots, q_out, cache, stream=0) == status


def test_append_refuses():
    for name in ("k", "v", "cos", "sin", "pos", "slots", "q_out", "cache"):
        _append(E.IFQ_EINVAL, **{name: None})
    for name in ("q", "k", "v", "q_out", "cache"):
        _append(E.IFQ_EALIGN, **{name: FAKE + 8})
    _append(E.IFQ_EALIGN, slots=FAKE + 4)
    _append(E.IFQ_EALIGN, pos=FAKE + 2)
    _append(E.IFQ_EINVAL, tokens=-1)
    _append(E.IFQ_EINVAL, dtype=ifq.IFQ_F32)
    _append(E.IFQ_EINVAL, rope=3)
    _append(E.IFQ_EINVAL, positions=0)
    _append(E.IFQ_EINVAL, q_heads=0)
    for rot in (0, 8, 40, 144, -16):
        _append(E.IFQ_ESHAPE, rot_dim=rot)
    _append(E.IFQ_EINVAL, q_stride=8 * 128 - 8)
    _append(E.IFQ_EINVAL, q_stride=8 * 128 + 4)
    _append(E.IFQ_EINVAL, k_stride=-8)
    _append(E.IFQ_EINVAL, v_stride=128)
    _append(E.IFQ_EUNSUPPORTED, pool=ifq.kv4_cache(2, 16, 2, 32))

def test_read_refuses():
    d = ifq.kv4_append_desc(ifq.kv4_cache(2, 16, 2, 128), 4, 8, ifq.IFQ_BF16)
    assert _status(ifq.ifq_kv4_read, d, None, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    assert _status(ifq.ifq_kv4_read, d, FAKE, None, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    assert _status(ifq.ifq_kv4_read, d, FAKE, FAKE, FAKE + 2, FAKE, stream=0) == E.IFQ_EALIGN
    d = ifq.kv4_append_desc(ifq.kv4_cache(2, 16, 2, 128), 4, 8, ifq.IFQ_F32)
    assert _status(ifq.ifq_kv4_read, d, FAKE, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL


def _attention(status, q=FAKE, cache=FAKE, table=FAKE, lens=FAKE, starts=FAKE, out=FAKE, lse=FAKE, ws=FAKE,
               ws_bytes=1 << 40, pool=None, **kw):
    a = dict(seqs=3, q_tokens=3, max_q=1, max_pages=4, q_heads=8, dtype=ifq.IFQ_BF16, scale=0.1)
    a.update(kw)
    d = ifq.kv4_attention_desc(pool or ifq.kv4_cache(2, 16, 2, 128), **a)
    assert _status(ifq.ifq_kv4_attention, d, q, cache, table, lens, starts, out, lse, ws, ws_bytes, stream=0) == status


def test_attention_refuses():
    for name in ("q", "cache", "table", "lens", "out"):
        _attention(E.IFQ_EINVAL, **{name: None})
    for name in ("q", "cache", "out", "ws"):
        _attention(E.IFQ_EALIGN, **{name: FAKE + 8})
    for name in ("table", "lens", "starts", "lse"):
        _attention(E.IFQ_EALIGN, **{name: FAKE + 2})
    for name in ("seqs", "q_tokens", "max_q", "max_pages", "max_len", "window", "sinks"):
        _attention(E.IFQ_EINVAL, **{name: -1})
    _attention(E.IFQ_EINVAL, scale=float("nan"))
    _attention(E.IFQ_EINVAL, scale=float("inf"))
    _attention(E.IFQ_EINVAL, dtype=ifq.IFQ_F32)
    _attention(E.IFQ_EINVAL, q_heads=0)
    _attention(E.IFQ_ESHAPE, q_heads=7)
    _attention(E.IFQ_ESHAPE, starts=None, q_tokens=4)
    _attention(E.IFQ_ERANGE, max_pages=2 ** 28)
    _attention(E.IFQ_EINVAL, q_stride=1016)
    _attention(E.IFQ_EINVAL, out_stride=1028)
    d = ifq.kv4_attention_desc(ifq.kv4_cache(2, 16, 2, 128), 3, 3, 1, 4, 7, ifq.IFQ_BF16, 0.1)
    assert _status(ifq.ifq_kv4_attention_workspace_bytes, d) == E.IFQ_ESHAPE


def _fp8(status, x=FAKE, xs=FAKE, w=FAKE, ws_=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
    a = dict(m=4, n=64, k=256)
    a.update(kw)
    d = ifq.fp8_desc(**a)
    assert _status(ifq.ifq_fp8_matmul, d, x, xs, w, ws_, out, ws, ws_bytes, stream=0) == status


def test_fp8_refuses():
    for name in ("x", "xs", "w", "ws_", "out"):
        _fp8(E.IFQ_EINVAL, **{name: None})
    for name in ("x", "w", "out", "ws"):
        _fp8(E.IFQ_EALIGN, **{name: FAKE + 8})
    for name in ("xs", "ws_"):
        _fp8(E.IFQ_EALIGN, **{name: FAKE + 2})
    _fp8(E.IFQ_EINVAL, m=-1)
    _fp8(E.IFQ_EINVAL, n=0)
    _fp8(E.IFQ_EINVAL, k=0)
    _fp8(E.IFQ_ESHAPE, k=24)
    _fp8(E.IFQ_EINVAL, out_dtype=4)
    _fp8(E.IFQ_EINVAL, out_stride=63)
    _fp8(E.IFQ_EINVAL, out_stride=-1)
    d = ifq.fp8_desc(4, 64, 256, ifq.IFQ_F32)
    assert _status(ifq.ifq_fp8_quantize, d, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    d = ifq.fp8_desc(4, 64, 256, x_stride=260)
    assert _status(ifq.ifq_fp8_quantize, d, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    d = ifq.fp8_desc(4, 64, 256)
    assert _status(ifq.ifq_fp8_quantize, d, FAKE, FAKE + 8, FAKE, stream=0) == E.IFQ_EALIGN
    assert _status(ifq.ifq_fp8_workspace_bytes, ifq.fp8_desc(4, 64, 250)) == E.IFQ_ESHAPE
