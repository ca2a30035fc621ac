"""Scores of tokens.  Ids are exact, numbers off by layer_reference.scores_tolerance."""
import numpy as np
import pytest
import torch

import layer_reference as R
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"f16": (ifq.IFQ_F16, torch.float16), "bf16": (ifq.IFQ_BF16, torch.bfloat16), "f32": (ifq.IFQ_F32, torch.float32)}


def run(logits, tokens, dtype, top, scale, stride=0, offset=0, expect=ifq.IFQ_OK):
    """logits float64 values of dtype [rows][vocab], placed in rows of `stride` from element `offset` on."""
    rows, vocab = logits.shape
    stride = stride or vocab
    flat = torch.full((offset + rows * stride + 64,), float("nan"), device=DEV, dtype=TYPES[dtype][1])
    flat[offset:offset + rows * stride].view(rows, stride)[:, :vocab] = torch.from_numpy(logits).to(DEV).to(TYPES[dtype][1])
    t = torch.as_tensor(tokens, dtype=torch.int64, device=DEV)
    f = lambda *s: torch.full(s, -7.0, device=DEV)                               # noqa: E731
    out = {"logprobs": f(rows + 1), "lse": f(rows + 1), "entropy": f(rows + 1),
           "top_ids": torch.full((rows + 1, top), -7, dtype=torch.int64, device=DEV), "top_logprobs": f(rows + 1, top)}
    d = ifq.scores_desc(rows, vocab, TYPES[dtype][0], top, scale, stride)
    ifq.ifq_token_scores(d, flat[offset:], t, *out.values())
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == expect
    assert all((v[rows:] == -7).all() for v in out.values())
    return {k: v[:rows].cpu().numpy() for k, v in out.items()}


def check(logits, tokens, dtype, top, scale, got):
    want = R.scores(logits, tokens, float(np.float32(scale)), top)
    assert np.array_equal(got["top_ids"], want["top_ids"])
    tol = R.scores_tolerance(logits, scale)
    for k in ("logprobs", "lse", "entropy", "top_logprobs"):
        t = tol[:, None] if k == "top_logprobs" else tol
        g, w = got[k].astype(np.float64), want[k]
        same = (g == w) | (np.isnan(g) & np.isnan(w))
        with np.errstate(invalid="ignore"):
            # (a token far from the likeliest: z itself is rounded, in the tolerance by the largest |z|)
            assert (same | (np.abs(g - w) <= t * (1 if k != "entropy" else 16))).all(), (k, np.nanmax(np.abs(g - w) / t))


def draw(rng, rows, vocab, dtype, spread=1.0):
    z = rng.normal(size=(rows, vocab)) * rng.uniform(0.5, 4, (rows, 1)) * spread
    return R.round_to(z, dtype)


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 31), (2, 33), (5, 100), (4, 1000), (1, 4097), (7, 32001), (2, 131072),
                                        (1, 131072), (1, 262144), (3, 262143), (40, 50257), (200, 5003), (700, 1024), (2000, 300)])
@pytest.mark.parametrize("dtype,top,scale", [("f32", 20, 1.25), ("bf16", 8, 1.0), ("f16", 32, 0.7), ("bf16", 0, 1.0), ("f32", 1, 1.0)])
def test_values(rows, vocab, dtype, top, scale):
    rng = np.random.default_rng([rows, vocab, top])
    top = min(top, vocab)
    logits, tokens = draw(rng, rows, vocab, dtype), rng.integers(0, vocab, rows)
    check(logits, tokens, dtype, top, scale, run(logits, tokens, dtype, top, scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("offset,more", [(1, 0), (3, 5), (7, 1), (0, 8), (5, 3), (2, 2)])
def test_rows_that_begin_anywhere(dtype, offset, more):
    rng = np.random.default_rng([offset, more])
    logits, tokens = draw(rng, 9, 2007, dtype), rng.integers(0, 2007, 9)
    logits[3, [0, 2006]] = 60.0       # the ends count
    check(logits, tokens, dtype, 6, 1.0, run(logits, tokens, dtype, 6, 1.0, 2007 + more, offset))


@pytest.mark.parametrize("vocab", [40, 3001, 65536, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_go_to_the_lowest_token(vocab, dtype):
    rng = np.random.default_rng(vocab)
    logits = np.zeros((8, vocab))
    logits[1] = rng.integers(0, 3, vocab)
    logits[2] = rng.integers(-1, 1, vocab) * 0.0            # zeros of both signs
    logits[3, vocab - 20:] = 1.0
    logits[4] = np.where(np.arange(vocab) % 2, 5.0, -5.0)
    logits[5] = np.minimum(np.arange(vocab), vocab // 2)    # rounds to many equals in bfloat16
    logits[6] = -np.arange(vocab)
    logits[7] = np.where(np.arange(vocab) == vocab - 1, 3.0, -1.0)
    more = np.zeros((6, vocab))
    more[0, rng.integers(0, vocab, 9)] = np.arange(9) + 1.0          # fewer above the many equals than wanted
    more[1] = -np.inf
    more[1, rng.integers(0, vocab, 5)] = 2.0
    more[2] = np.where(np.arange(vocab) >= vocab - vocab // 3, 2.0, np.arange(vocab) / vocab)   # equals at the end
    more[3] = np.where(np.arange(vocab) % 64 == 63, 4.0, -4.0)
    more[4, : vocab // 2] = np.linspace(1, 2, vocab // 2)            # many above, and equals
    more[5, rng.random(vocab) < 0.3] = np.nan
    logits = np.concatenate([logits, more])
    logits = R.round_to(logits, dtype)
    tokens = rng.integers(0, vocab, 14)
    for top in (1, 7, 32):
        check(logits, tokens, dtype, top, 0.01, run(logits, tokens, dtype, top, 0.01))


@pytest.mark.parametrize("vocab", [37, 5000, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masked_and_infinite_logits(vocab, dtype):
    rng = np.random.default_rng(vocab)
    logits = draw(rng, 9, vocab, dtype)
    logits[0, rng.random(vocab) < 0.9] = -np.inf
    logits[1] = -np.inf
    logits[2] = -np.inf
    logits[2, vocab // 2] = -3.0                              # one token left
    logits[3, vocab - 1] = np.inf
    logits[4, [1, vocab // 3]] = np.nan
    logits[5, 0], logits[5, 2] = np.nan, np.inf
    logits[6] = 60000.0 if dtype == "f16" else 1e30
    logits[7] = -60000.0 if dtype == "f16" else -1e30
    logits[8, 1:] = -np.inf
    logits = R.round_to(logits, dtype)
    tokens = rng.integers(0, vocab, 9)
    got = run(logits, tokens, dtype, 5, 1.0)
    check(logits, tokens, dtype, 5, 1.0, got)
    assert got["entropy"][2] == 0 and got["lse"][1] == -np.inf


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [1.0, 1e-4, 1e-6, 30.0])
@pytest.mark.parametrize("vocab", [300, 20011])
def test_masks_of_the_lowest_value_beside_infinities(vocab, dtype, scale):
    """A finite mask counts by its value, however hot the temperature; -infinity never does."""
    rng = np.random.default_rng(vocab)
    lowest = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38, "f16": -65504.0}[dtype]
    logits = draw(rng, 7, vocab, dtype)
    logits[0, rng.random(vocab) < 0.7] = lowest
    logits[1] = lowest
    logits[2, rng.random(vocab) < 0.7] = -np.inf
    logits[3] = lowest
    logits[3, ::3] = -np.inf
    logits[4] = -np.inf
    logits[4, vocab - 1] = lowest
    logits[5, ::2], logits[5, 1::4] = -np.inf, lowest
    logits[6] = -lowest
    tokens = rng.integers(0, vocab, 7)
    got = run(logits, tokens, dtype, 3, scale)
    want = R.scores(logits, tokens, float(np.float32(scale)), 3)
    tol = R.scores_tolerance(np.where(logits < lowest / 2, 0, logits), scale)
    assert np.array_equal(got["top_ids"], want["top_ids"])
    for k in ("entropy", "logprobs", "lse"):
        with np.errstate(invalid="ignore", over="ignore"):
            w = want[k].astype(np.float32).astype(np.float64)     # (what a float cannot hold is infinite)
            close = np.abs(got[k] - w) <= 16 * tol + np.abs(w) * 2.0 ** -22
        assert (close | (got[k] == w)).all(), (k, got[k], w)


def test_tokens_outside_the_vocabulary():
    rng = np.random.default_rng(3)
    logits, tokens = draw(rng, 5, 700, "f32"), [-1, 699, 700, 0, 2 ** 40]
    got = run(logits, tokens, "f32", 2, 1.0, expect=ifq.IFQ_ERANGE)
    check(logits, tokens, "f32", 2, 1.0, got)
    run(logits, [-1, -2 ** 40, 0, 1, 2], "f32", 2, 1.0)


@pytest.mark.parametrize("rows,vocab", [(1, 131072), (300, 2000)])
def test_outputs_that_are_not_wanted(rows, vocab):
    rng = np.random.default_rng(4)
    logits, tokens = draw(rng, rows, vocab, "bf16"), rng.integers(0, vocab, rows)
    full = run(logits, tokens, "bf16", 4, 1.0)
    x = torch.from_numpy(logits).to(DEV).bfloat16()
    d = ifq.scores_desc(rows, vocab, ifq.IFQ_BF16, 4)
    for name in full:
        out = torch.empty(full[name].shape, dtype=torch.int64 if name == "top_ids" else torch.float32, device=DEV)
        t = torch.from_numpy(tokens).to(DEV) if name == "logprobs" else None
        ifq.ifq_token_scores(d, x, t, **{name: out})
        assert np.array_equal(out.cpu().numpy(), full[name]), name


@pytest.mark.parametrize("rows,vocab,top", [(1, 131072, 20), (64, 30001, 5), (900, 5000, 3)])
def test_same_bits_in_every_call_on_any_stream_and_in_graphs(rows, vocab, top):
    rng = np.random.default_rng(rows)
    x = torch.from_numpy(draw(rng, rows, vocab, "bf16")).to(DEV).bfloat16()
    t = torch.from_numpy(rng.integers(0, vocab, rows)).to(DEV)
    d = ifq.scores_desc(rows, vocab, ifq.IFQ_BF16, top)

    def once():
        o = [torch.empty(rows, device=DEV) for _ in range(3)]
        o += [torch.empty(rows, top, dtype=torch.int64, device=DEV), torch.empty(rows, top, device=DEV)]
        ifq.ifq_token_scores(d, x, t, *o)
        return o

    want = [v.clone() for v in once()]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for i in range(9):
        with torch.cuda.stream(streams[i % 3]):
            got.append(once())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = once()
    for _ in range(2):
        for v in o:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got.append([v.clone() for v in o])
    assert all(torch.equal(p, q) for one in got for p, q in zip(one, want))


def test_rows_past_32_bits():
    """Rows that begin past 2^31 elements."""
    vocab, rows = 1 << 20, 2100
    x = torch.zeros(rows, vocab, dtype=torch.float16, device=DEV)
    x[rows - 1, 77777] = 4.0
    lse, ids = torch.empty(rows, device=DEV), torch.empty(rows, 1, dtype=torch.int64, device=DEV)
    ifq.ifq_token_scores(ifq.scores_desc(rows, vocab, ifq.IFQ_F16, 1), x, None, lse=lse, top_ids=ids)
    assert ids[-1].item() == 77777 and not ids[:-1].any()
    tol = 2.0 ** -22 * 12 + (vocab / 256 + 32) * 2.0 ** -24
    assert abs(lse[0].item() - np.log(vocab)) < tol * 2 and abs(lse[-1].item() - np.log(vocab - 1 + np.exp(4.0))) < tol * 2
