"""Scores of tokens beside other work.  Ids are exact, numbers off by layer_reference.scores_tolerance."""
import numpy as np
import pytest
import torch

import layer_reference as R
from paper_1911_08076_gb300 import ifq
from test_gpu_scores import TYPES, check, draw, run

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131072, "f32"), (1, 262143, "bf16"), (48, 50257, "bf16"), (3, 100003, "f16")])
@pytest.mark.parametrize("top", [1, 5, 20, 32])
def test_split_rows_beside_another_stream(rows, vocab, dtype, top):
    """A row's parts run at different paces: another stream's blocks come and go on the SMs, and its copies fill the memory.
    Every call's tokens are the definition's, and its bits the first call's."""
    rng = np.random.default_rng([rows, vocab, top])
    logits, tokens = draw(rng, rows, vocab, dtype), rng.integers(0, vocab, rows)
    x, t = torch.from_numpy(logits).to(DEV).to(TYPES[dtype][1]), torch.from_numpy(tokens).to(DEV)
    d = ifq.scores_desc(rows, vocab, TYPES[dtype][0], top)

    def once():
        o = [torch.full((rows,), -7.0, device=DEV) for _ in range(3)]
        o += [torch.full((rows, top), -7, dtype=torch.int64, device=DEV), torch.full((rows, top), -7.0, device=DEV)]
        ifq.ifq_token_scores(d, x, t, *o)
        return o

    busy = torch.cuda.Stream()
    small = [torch.zeros(1 << n, device=DEV) for n in (12, 16, 20)]
    big, to = torch.zeros(1 << 26, device=DEV), torch.empty(1 << 26, device=DEV)
    want = R.scores(logits, tokens, 1.0, top)
    torch.cuda.synchronize()
    got = []
    for i in range(60):
        with torch.cuda.stream(busy):
            if i % 4 == 0:
                to.copy_(big)
            for s in small:
                s.add_(1.0)
        got.append(once())
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
    tol = R.scores_tolerance(logits, 1.0)
    for o in got:
        assert np.array_equal(o[3].cpu().numpy(), want["top_ids"])
        assert all(torch.equal(a, b) for a, b in zip(o, got[0]))
    assert (np.abs(got[0][1].cpu().numpy() - want["lse"]) <= tol).all()
    assert (np.abs(got[0][4].cpu().numpy() - want["top_logprobs"]) <= tol[:, None]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,top", [(300, 5), (70001, 8)])
@pytest.mark.parametrize("scale", [1e-38, 2.0 ** -127, 1e-37])
def test_logits_farther_apart_than_a_float_holds(vocab, top, dtype, scale):
    """Differences of logits past 2^128, which a small scale brings back into range."""
    rng = np.random.default_rng(vocab)
    logits = rng.uniform(-3.38e38, 3.38e38, (5, vocab))
    logits[1] = np.where(rng.random(vocab) < 0.9, -3.38e38, 3e38)
    logits[2], logits[2, vocab // 2] = -3.38e38, 3.38e38
    logits[3, ::3] = -np.inf
    logits[4] = rng.normal(size=vocab) * 1e37
    logits = R.round_to(logits, dtype)
    tokens = rng.integers(0, vocab, 5)
    check(logits, tokens, dtype, top, scale, run(logits, tokens, dtype, top, scale))
