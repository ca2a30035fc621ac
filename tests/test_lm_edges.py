"""Calls of the decoder's operators that have nothing to do, or sizes at the ends of their ranges (no GPU)."""
import pytest
import torch

from paper_1911_08076_gb300 import decoder, ifq

FAKE = 1 << 20     # never dereferenced


def test_calls_without_rows_take_null_pointers():
    """An empty tensor's address is 0."""
    pool = ifq.kv4_cache(2, 16, 2, 128)
    d = ifq.kv4_append_desc(pool, 0, 8, ifq.IFQ_BF16, positions=10)
    ifq.ifq_kv4_append(d, None, None, None, FAKE, FAKE, None, None, None, FAKE, stream=0)
    ifq.ifq_kv4_read(d, FAKE, None, None, None, stream=0)
    for seqs, starts in ((3, FAKE), (0, FAKE), (0, None)):
        d = ifq.kv4_attention_desc(pool, seqs, 0, 0, 4, 8, ifq.IFQ_BF16, 0.1)
        ifq.ifq_kv4_attention(d, None, FAKE, FAKE if seqs else None, FAKE if seqs else None, starts, None, None, None, 0, stream=0)
    d = ifq.fp8_desc(0, 64, 256)
    ifq.ifq_fp8_quantize(d, None, None, None, stream=0)
    ifq.ifq_fp8_matmul(d, None, None, FAKE, FAKE, None, None, 0, stream=0)


def test_calls_without_rows_still_refuse_their_descriptors():
    for f, d in ((ifq.ifq_fp8_quantize, ifq.fp8_desc(0, 64, 24)), (ifq.ifq_fp8_quantize, ifq.fp8_desc(0, 64, 32, ifq.IFQ_F32)),
                 (ifq.ifq_fp8_quantize, ifq.fp8_desc(0, 64, 32, x_stride=20))):
        with pytest.raises(ifq.IfqError):
            f(d, None, None, None, stream=0)
    with pytest.raises(ifq.IfqError):
        ifq.ifq_fp8_matmul(ifq.fp8_desc(0, 64, 32, out_dtype=9), None, None, FAKE, FAKE, None, None, 0, stream=0)
    pool = ifq.kv4_cache(2, 24, 2, 128)
    with pytest.raises(ifq.IfqError):
        ifq.ifq_kv4_read(ifq.kv4_append_desc(pool, 0, 8, ifq.IFQ_BF16), FAKE, None, None, None, stream=0)
    with pytest.raises(ifq.IfqError):
        ifq.ifq_kv4_attention(ifq.kv4_attention_desc(ifq.kv4_cache(2, 16, 2, 128), 3, 0, 0, 4, 7, ifq.IFQ_BF16, 0.1), None, FAKE,
                              FAKE, FAKE, FAKE, None, stream=0)
    with pytest.raises(ifq.IfqError):      # without starts each sequence has a row
        ifq.ifq_kv4_attention(ifq.kv4_attention_desc(ifq.kv4_cache(2, 16, 2, 128), 3, 0, 0, 4, 8, ifq.IFQ_BF16, 0.1), None, FAKE,
                              FAKE, FAKE, None, None, stream=0)


@pytest.mark.parametrize("seqs", [0, 2])
def test_a_step_without_tokens(monkeypatch, seqs):
    monkeypatch.setattr(ifq, "_stream", lambda stream: 0)
    block = decoder.DecoderAttention(torch.randn(256, 64), torch.randn(64, 128), 2, 1, 64, 8, 16, 64)
    pages = decoder.PagedSequences(8, 16, device="cpu")
    step = pages.extend([pages.add() for _ in range(seqs)], [0] * seqs)
    assert block.forward(torch.zeros(0, 64, dtype=torch.bfloat16), step).shape == (0, 64)


def test_a_stride_of_q_does_not_count_without_q():
    pool = ifq.kv4_cache(2, 16, 2, 128)
    for stride in (0, 8, 1000, 1024, 12):
        for q_out in (0, 8):
            d = ifq.kv4_append_desc(pool, 0, 8, ifq.IFQ_BF16, ifq.IFQ_ROPE_NONE, q_stride=stride, q_out_stride=q_out)
            ifq.ifq_kv4_append(d, None, FAKE, FAKE, None, None, None, FAKE, None, FAKE, stream=0)
    d = ifq.kv4_append_desc(pool, 0, 8, ifq.IFQ_BF16, ifq.IFQ_ROPE_NONE, q_stride=8)
    with pytest.raises(ifq.IfqError):
        ifq.ifq_kv4_append(d, FAKE, FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, stream=0)


def _status(f, *a, **k):
    with pytest.raises(ifq.IfqError) as e:
        f(*a, **k)
    return e.value.status


def test_sizes_that_end_past_31_bits():
    """Sizes so near 2^31 that the end of a last block would lie past it are refused, not wrapped."""
    top = 2 ** 31 - 1
    for m, n, k in ((top, 8, 16), (8, top, 16), (8, 8, 2 ** 31 - 16), (top - 1022, 8, 16)):
        d = ifq.fp8_desc(m, n, k)
        assert _status(ifq.ifq_fp8_matmul, d, FAKE, FAKE, FAKE, FAKE, FAKE, stream=0) == ifq.IFQ_ERANGE
        assert _status(ifq.ifq_fp8_quantize, d, FAKE, FAKE, FAKE, stream=0) == ifq.IFQ_ERANGE
        assert _status(ifq.ifq_fp8_workspace_bytes, d) == ifq.IFQ_ERANGE
    assert ifq.ifq_fp8_workspace_bytes(ifq.fp8_desc(top - 1023, top - 1023, 2 ** 31 - 1024)) == 0
    pool = ifq.kv4_cache(2, 16, 2, 128)
    d = ifq.kv4_append_desc(pool, top, 2, ifq.IFQ_BF16, ifq.IFQ_ROPE_NONE)
    assert _status(ifq.ifq_kv4_append, d, None, FAKE, FAKE, None, None, None, FAKE, None, FAKE, stream=0) == ifq.IFQ_ERANGE
    assert _status(ifq.ifq_kv4_read, d, FAKE, FAKE, FAKE, FAKE, stream=0) == ifq.IFQ_ERANGE
    ok = dict(seqs=2, q_tokens=2, max_q=1, max_pages=4, q_heads=8, dtype=ifq.IFQ_BF16, scale=0.1)
    for name, value in (("seqs", top), ("q_tokens", top), ("max_pages", 2 ** 27 - 1), ("max_q", top // 8), ("max_len", top)):
        d = ifq.kv4_attention_desc(pool, **{**ok, name: value})
        want = ifq.IFQ_OK if name == "max_len" else ifq.IFQ_ERANGE     # (a bound of any size says nothing)
        if want:
            assert _status(ifq.ifq_kv4_attention_workspace_bytes, d) == want
        else:
            ifq.ifq_kv4_attention_workspace_bytes(d)
    ifq.ifq_kv4_attention_workspace_bytes(ifq.kv4_attention_desc(pool, **{**ok, "max_pages": 2 ** 27 - 64}))
