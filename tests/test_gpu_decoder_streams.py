"""Steps of one decoder block on two streams at once, and captured steps replayed after others."""
import pytest
import torch

from paper_1911_08076_gb300 import decoder, ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _block(pages, page, hidden=256, hq=8, hk=2, d=64):
    torch.manual_seed(2)
    return decoder.DecoderAttention(torch.randn((hq + 2 * hk) * d, hidden, device=DEV) * hidden ** -0.5,
                                    torch.randn(hidden, hq * d, device=DEV) * (hq * d) ** -0.5, hq, hk, d, pages, page, 1024)


def _x(n, seed):
    return torch.randn(n, 256, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).bfloat16()


def test_two_streams():
    block, seqs = _block(128, 16), decoder.PagedSequences(128, 16)
    halves = [[seqs.add() for _ in range(3)] for _ in range(2)]
    steps = [[seqs.extend(h, c) for c in ([60, 200, 1], [1, 1, 1], [4, 30, 2], [1, 1, 1])] for h in halves]
    xs = [[_x(s.positions.numel(), 10 * i + j) for j, s in enumerate(h)] for i, h in enumerate(steps)]
    want = [[block.forward(x, s).clone() for x, s in zip(xs[i], steps[i])] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        block.cache.zero_()
        torch.cuda.synchronize()
        got = [[], []]
        for j in range(4):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    got[i].append(block.forward(xs[i][j], steps[i][j]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    assert ifq.ifq_device_status() == ifq.IFQ_OK


def test_a_captured_step_after_a_larger_one():
    block, seqs = _block(128, 16), decoder.PagedSequences(128, 16)
    a, b = seqs.add(), seqs.add()
    block.forward(_x(70, 1), seqs.extend([a], [70]))
    step, x = seqs.extend([a], [1]), _x(1, 2)
    want = block.forward(x, step).clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = block.forward(x, step)
    big = block.forward(_x(900, 3), seqs.extend([b], [900])).clone()
    torch.cuda.empty_cache()
    fill = [torch.full((1 << 20,), 3, dtype=torch.uint8, device=DEV) for _ in range(20)]
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    assert all((f == 3).all() for f in fill) and torch.isfinite(big).all()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
