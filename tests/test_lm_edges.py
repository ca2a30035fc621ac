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
