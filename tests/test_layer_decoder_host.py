"""What decoder.py's feed-forward, norm and scores give their calls, and what they refuse (no GPU): the calls that launch
kernels are replaced by ones that note their arguments."""
import pytest
import torch

from paper_1911_08076_gb300 import decoder, ifq


@pytest.fixture
def calls(monkeypatch):
    seen = []
    for name in ("ifq_w4_pack", "ifq_w4_matmul", "ifq_w4_gated", "ifq_rms_norm", "ifq_token_scores", "ifq_fp8_quantize",
                 "ifq_fp8_matmul", "ifq_kv4_append", "ifq_kv4_attention"):
        monkeypatch.setattr(ifq, name, lambda *a, _name=name, **k: seen.append((_name, a)))
    return seen


def test_codes_and_parameters_by_hand():
    w = torch.zeros(2, 40)
    w[0, :32] = torch.arange(32) * 0.25 - 1.0      # -1 ... 6.75 in 15 steps of 31/60
    w[0, 32:] = 3.0                                # one value: scale 0
    codes, scales, mins = decoder.quantise_weights4(w, 32)
    assert codes.shape == (2, 20) and codes.dtype == torch.uint8 and scales.shape == mins.shape == (2, 2)
    assert mins[0].tolist() == [-1.0, 3.0] and scales[0, 1] == 0 and scales[0, 0] == torch.tensor(7.75 / 15).bfloat16()
    assert codes[0, 0] == 0 and codes[0, 15] >> 4 == 15 and (codes[0, 16:] == 0).all() and (codes[1] == 0).all()


def test_a_layer_calls_in_order(calls):
    hidden, inner = 64, 48
    attention = decoder.DecoderAttention(torch.randn(4 * 64, hidden), torch.randn(hidden, 2 * 64), 2, 1, 64, 8, 16, 64)
    ff = decoder.FeedForward(torch.randn(inner, hidden), torch.randn(inner, hidden), torch.randn(hidden, inner), "gelu", 32)
    layer = decoder.DecoderLayer(attention, ff, torch.ones(hidden), torch.ones(hidden), 1e-6)
    assert [n for n, _ in calls] == ["ifq_w4_pack", "ifq_w4_pack"]
    assert calls[0][1][0].gated == 1 and calls[0][1][1].shape == (2 * inner, hidden // 2) and calls[1][1][0].gated == 0
    del calls[:]
    seqs = decoder.PagedSequences(8, 16, device="cpu")
    x = torch.zeros(5, hidden, dtype=torch.bfloat16)
    y = layer.forward(x, seqs.extend([seqs.add()], [5]))
    assert [n for n, _ in calls] == ["ifq_rms_norm", "ifq_fp8_quantize", "ifq_fp8_matmul", "ifq_kv4_append", "ifq_kv4_attention",
                                     "ifq_fp8_quantize", "ifq_fp8_matmul", "ifq_rms_norm", "ifq_w4_gated", "ifq_w4_matmul"]
    norm1, norm2, gated, down = calls[0][1], calls[7][1], calls[8][1], calls[9][1]
    assert norm1[1] is x and norm1[2] is None and norm1[4] is None and abs(norm1[0].eps - 1e-6) < 1e-12
    assert norm2[2] is x and norm2[4] is not None and gated[1] is norm2[5] and gated[0].act == ifq.IFQ_ACT_GELU
    assert down[1] is gated[3] and down[4] is norm2[4] and down[3] is y and y.shape == x.shape
    # a step's buffers are its own
    first = {t.data_ptr() for _, a in calls for t in (a[-1],) if isinstance(t, torch.Tensor)}
    held = list(calls)
    del calls[:]
    layer.forward(x, seqs.extend([seqs.add()], [5]))
    again = {a[5].data_ptr() for n, a in calls if n == "ifq_rms_norm"} | {a[3].data_ptr() for n, a in calls if n.startswith("ifq_w4")}
    before = {a[5].data_ptr() for n, a in held if n == "ifq_rms_norm"} | {a[3].data_ptr() for n, a in held if n.startswith("ifq_w4")}
    assert not again & before and first


def test_strided_rows_and_scores(calls):
    w = decoder.Weights4(torch.randn(24, 40), group=32)
    wide = torch.zeros(6, 64, dtype=torch.bfloat16)
    w.matmul(wide[:, :40], out_dtype=torch.float32)
    assert calls[-1][1][0].x_stride == 64 and calls[-1][1][0].out_dtype == ifq.IFQ_F32
    s = decoder.token_scores(torch.zeros(3, 50, dtype=torch.float16)[:, :33], torch.zeros(3, dtype=torch.int64), 4, 0.5)
    d = calls[-1][1][0]
    assert (d.vocab, d.stride, d.top, d.scale, d.dtype) == (33, 50, 4, 2.0, ifq.IFQ_F16) and s.top_ids.shape == (3, 4)
    s = decoder.token_scores(torch.zeros(2, 33))
    assert s.logprobs is None and s.top_ids is None and calls[-1][1][2] is None and calls[-1][1][3] is None


def test_refusals(calls):
    w = decoder.Weights4(torch.randn(24, 40), group=32)
    x = torch.zeros(6, 40, dtype=torch.bfloat16)
    for bad in (x.float(), x[:, :32], x.t().contiguous().t(), torch.zeros(6, 44, dtype=torch.bfloat16)[:, :40], x[0]):
        with pytest.raises(ValueError):
            w.matmul(bad)
    for bad in (torch.zeros(6, 23, dtype=torch.bfloat16), torch.zeros(6, 24), torch.zeros(6, 48, dtype=torch.bfloat16)[:, :24]):
        with pytest.raises(ValueError):
            w.matmul(x, bad)
    with pytest.raises(ValueError):
        decoder.Weights4(torch.randn(24, 40), torch.randn(24, 48))
    with pytest.raises(ValueError):
        decoder.FeedForward(torch.randn(24, 40), torch.randn(24, 40), torch.randn(40, 32))
    with pytest.raises(ifq.IfqError):
        decoder.Weights4(torch.randn(24, 44))                       # k is a multiple of 8
    weight = torch.ones(40, dtype=torch.bfloat16)
    for a in ((x.float(), weight), (x, weight[:32]), (x, weight, 1e-5, x[:3]), (x, weight, 1e-5, x.float()), (x[:, ::2], weight[::2])):
        with pytest.raises(ValueError):
            decoder.rms_norm(*a)
    for a in ((x[0],), (x, torch.zeros(6, dtype=torch.int32)), (x, torch.zeros(5, dtype=torch.int64)), (x.t(),)):
        with pytest.raises(ValueError):
            decoder.token_scores(*a)
