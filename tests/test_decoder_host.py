"""The decoder block's host side (no GPU): what its calls are given.  The calls that launch kernels are replaced by ones
that note their arguments."""
import pytest
import torch

from paper_1911_08076_gb300 import decoder, ifq


@pytest.fixture
def calls(monkeypatch):
    """The arguments of every launching call, in order: (name, arguments)."""
    seen = []
    for name in ("ifq_fp8_quantize", "ifq_fp8_matmul", "ifq_kv4_append", "ifq_kv4_attention"):
        monkeypatch.setattr(ifq, name, lambda *a, _name=name, **k: seen.append((_name, a)))
    return seen


def _block(hidden=64, hq=2, hk=1, d=64, pages=8, page=16, positions=64, **kw):
    torch.manual_seed(1)
    return decoder.DecoderAttention(torch.randn((hq + 2 * hk) * d, hidden), torch.randn(hidden, hq * d), hq, hk, d, pages,
                                    page, positions, **kw)


@pytest.fixture
def default_dtype():
    was = torch.get_default_dtype()
    yield torch.set_default_dtype
    torch.set_default_dtype(was)


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_scales_are_float_whatever_the_default_type(calls, default_dtype, default):
    """The library reads and writes scales as floats: a buffer of a 16-bit default type would be half as large."""
    w = torch.randn(130, 272)
    codes, scales = decoder.quantise_weights(w)
    default_dtype(default)
    codes2, scales2 = decoder.quantise_weights(w)
    assert scales2.dtype == torch.float32 and torch.equal(scales, scales2)
    assert torch.equal(codes.view(torch.uint8), codes2.view(torch.uint8))
    block, seqs = _block(), decoder.PagedSequences(8, 16, device="cpu")
    block.forward(torch.zeros(5, 64, dtype=torch.bfloat16), seqs.extend([seqs.add()], [5]))
    assert block.s_qkv.dtype == block.s_out.dtype == block.cos.dtype == block.sin.dtype == torch.float32
    for name, a in calls:
        if name == "ifq_fp8_quantize":
            assert a[3].dtype == torch.float32 and a[3].numel() == -(-a[0].k // 128) * 5
        if name == "ifq_fp8_matmul":
            assert a[2].dtype == a[4].dtype == torch.float32


def test_steps_share_no_buffers(calls):
    """Two steps may be under way on two streams, and a captured one is replayed after a larger one: what a step writes
    belongs to it alone (but for the cache)."""
    block, seqs = _block(window=8), decoder.PagedSequences(8, 16, device="cpu")
    ids = [seqs.add(), seqs.add()]
    held = []
    for n in (3, 3, 40, 3):
        step = seqs.extend(ids[:1] if n == 3 else ids[1:], [n])
        x = torch.zeros(n, 64, dtype=torch.bfloat16)
        first = len(calls)
        y = block.forward(x, step)
        own = [y] + [t for _, a in calls[first:] for t in a[1:] if isinstance(t, torch.Tensor)]
        shared = {t.untyped_storage().data_ptr() for t in (block.w_qkv, block.s_qkv, block.w_out, block.s_out, block.cos,
                                                           block.sin, block.cache)}
        held.append((own, {t.untyped_storage().data_ptr() for t in own if t.numel()} - shared))
    for i, (_, a) in enumerate(held):
        for _, b in held[:i]:
            assert not a & b


def test_a_step_that_the_block_has_no_positions_or_pages_for_is_refused(calls):
    block = _block(pages=8, page=16, positions=48)
    run = lambda seqs, s, n: block.forward(torch.zeros(n, 64, dtype=torch.bfloat16), seqs.extend([s], [n]))   # noqa: E731
    seqs = decoder.PagedSequences(8, 16, device="cpu")
    a, b = seqs.add(), seqs.add()
    run(seqs, a, 47)
    run(seqs, a, 1)              # position 47, the last
    before = len(calls)
    for s, n in ((a, 1), (b, 49)):
        with pytest.raises(ValueError, match="position"):
            run(seqs, s, n)
    for other in (decoder.PagedSequences(9, 16, device="cpu"), decoder.PagedSequences(8, 32, device="cpu")):
        with pytest.raises(ValueError, match="page"):
            run(other, other.add(), 1)
    assert len(calls) == before
    fewer = decoder.PagedSequences(7, 16, device="cpu")
    run(fewer, fewer.add(), 1)
    # without a rotation there are no tables to run past
    block = _block(pages=8, page=16, positions=48, rope=ifq.IFQ_ROPE_NONE)
    seqs = decoder.PagedSequences(8, 16, device="cpu")
    run(seqs, seqs.add(), 60)
