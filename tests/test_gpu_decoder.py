"""The attention block of a quantised decoder (decoder.py): every stage of a prompt and of the steps after it against the
references, from the stage's own inputs."""
import numpy as np
import pytest
import torch

import lm_reference as R
from paper_1911_08076_gb300 import decoder, ifq

DEV = "cuda"


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hk,d,dtype,window,sinks", [(8, 2, 64, torch.bfloat16, 0, 0), (4, 1, 128, torch.float16, 24, 3)])
def test_prompt_and_steps(hq, hk, d, dtype, window, sinks):
    torch.manual_seed(0)
    hidden, page = 272, 16
    w_qkv = torch.randn((hq + 2 * hk) * d, hidden, device=DEV) * hidden ** -0.5
    w_out = torch.randn(hidden, hq * d, device=DEV) * (hq * d) ** -0.5
    block = decoder.DecoderAttention(w_qkv, w_out, hq, hk, d, 24, page, 256, dtype, window=window, sinks=sinks)
    seqs = decoder.PagedSequences(24, page)
    ids = [seqs.add() for _ in range(3)]
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    stale = seqs.extend(ids[:1], [30])      # pages that another conversation leaves behind
    block.forward(torch.randn(30, hidden, device=DEV).to(dtype) * 3, stale)
    seqs.release(ids[0])
    for counts in ([70, 1, 33], [1, 1, 1], [1, 0, 1], [5, 2, 3]):
        step = seqs.extend(ids, counts)
        x = torch.randn(sum(counts), hidden, device=DEV).to(dtype)
        before = block.cache.clone()
        y = block.forward(x, step)
        torch.cuda.synchronize()
        assert ifq.ifq_device_status() == ifq.IFQ_OK
        num = lambda t: t.float().cpu().numpy()   # noqa: E731

        def product(inp, w, s, out):
            xq, xs = R.fp8_quantise(num(inp))
            want, mag = R.fp8_matmul(xq, xs, w.view(torch.uint8).cpu().numpy(), s.cpu().numpy())
            tol = u * np.abs(want) + 2 * (128 + xs.shape[0]) * 2.0 ** -24 * mag
            assert (np.abs(num(out) - want) <= tol).all()

        product(x, block.w_qkv, block.s_qkv, block.qkv)
        # the rotation and the cache, byte by byte
        pos, slots = step.positions.cpu().numpy(), step.slots.cpu().numpy()
        qkv = num(block.qkv).reshape(len(pos), hq + 2 * hk, d)
        c, sn = block.cos.cpu().numpy()[pos], block.sin.cpu().numpy()[pos]
        kr = R.rotate(qkv[:, hq:hq + hk], c, sn, "halves", d)
        want = before.cpu().numpy().reshape(24, hk, page // 16, R.group_bytes(d))
        for t in range(len(pos)):
            for h in range(hk):
                R.write(want, page, slots[t], h, d, R.quantise4(kr[t, h]), R.quantise4(qkv[t, hq + hk + h]))
        assert np.array_equal(block.cache.cpu().numpy().reshape(want.shape), want)
        q = R.rotate(qkv[:, :hq], c, sn, "halves", d).reshape(len(pos), -1)
        q = R.to_bf16(q) if dtype == torch.bfloat16 else q.astype(np.float16).astype(np.float32)
        assert np.array_equal(num(block.q), q)
        out, _, tol, _ = R.attention(q.astype(np.float64).reshape(len(pos), hq, d), want, page, step.table.cpu().numpy(),
                                     step.lens.cpu().numpy(), step.starts.cpu().numpy(), hk, d ** -0.5, window, sinks, u,
                                     dtype == torch.bfloat16 and max(counts) * (hq // hk) > 32)
        assert (np.abs(num(block.context).reshape(out.shape) - out) <= tol).all()
        product(block.context, block.w_out, block.s_out, y)


def test_page_bookkeeping():
    s = decoder.PagedSequences(4, 16, device="cpu")
    a, b = s.add(), s.add()
    st = s.extend([a, b], [17, 3])
    assert st.lens.tolist() == [17, 3] and st.starts.tolist() == [0, 17, 20] and (st.max_q, st.max_len) == (17, 17)
    assert st.positions.tolist() == list(range(17)) + [0, 1, 2]
    pages = st.table.tolist()
    assert len({pages[0][0], pages[0][1], pages[1][0]}) == 3
    assert st.slots[16] == pages[0][1] * 16 and st.slots[17] == pages[1][0] * 16
    st = s.extend([b], [0])
    assert st.positions.numel() == 0 and st.lens.tolist() == [3]
    with pytest.raises(MemoryError):
        s.extend([b], [40])
    with pytest.raises(ValueError):
        s.extend([a, a], [1, 1])
    assert s.length == [17, 3] and len(s.free) == 1
    s.release(a)
    assert s.length == [0, 3] and len(s.free) == 3
    assert s.extend([a, b], [16, 13]).lens.tolist() == [16, 16]
