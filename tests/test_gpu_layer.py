"""A decoder layer and its head, run as they would be: every stage against the references from the stage's own inputs."""
import numpy as np
import pytest
import torch

import layer_reference as R
from paper_1911_08076_gb300 import decoder, ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"


def num(t):
    return t.double().cpu().numpy()


def layer_of(hidden, inner, hq, hk, d, dtype, group, act="silu"):
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)   # noqa: E731
    attention = decoder.DecoderAttention(r((hq + 2 * hk) * d, hidden) * hidden ** -0.5, r(hidden, hq * d) * (hq * d) ** -0.5, hq, hk,
                                         d, 48, 16, 512, dtype)
    raw = [r(inner, hidden) * hidden ** -0.5, r(inner, hidden) * hidden ** -0.5, r(hidden, inner) * inner ** -0.5]
    ff = decoder.FeedForward(*raw, act=act, group=group, dtype=dtype)
    return decoder.DecoderLayer(attention, ff, 1 + 0.1 * r(hidden), 1 + 0.1 * r(hidden)), raw


@pytest.mark.parametrize("group,dtype", [(32, torch.float16), (64, torch.bfloat16), (128, torch.bfloat16)])
def test_weights_keep_to_half_a_step(group, dtype):
    """A weight is off by half a step of its group (15 of which are the range), and by what the roundings of scale, minimum and
    value add: a scale's is multiplied by 15."""
    w = torch.randn(40, 200, device=DEV) * torch.linspace(0.01, 3, 40, device=DEV)[:, None]
    w[3], w[4, :100] = 0.25, -1.5
    codes, scales, mins = decoder.quantise_weights4(w, group, dtype)
    name = "f16" if dtype == torch.float16 else "bf16"
    v = R.weights(codes.cpu().numpy(), num(scales), num(mins), group, name)
    at = np.arange(200) // group
    s, m, u = num(scales)[:, at], num(mins)[:, at], R.half_step(name)
    assert (np.abs(v - num(w)) <= 0.5 * s + u * (15 * s + 2 * np.abs(m) + np.abs(v)) * (1 + 1e-3) + 1e-7).all()


@pytest.mark.parametrize("hidden,inner,dtype,group,act", [(256, 520, torch.bfloat16, 64, "silu"), (272, 264, torch.float16, 32, "gelu_tanh")])
def test_layer_stage_by_stage(hidden, inner, dtype, group, act):
    layer, raw = layer_of(hidden, inner, 4, 2, 64, dtype, group, act)
    name = "f16" if dtype == torch.float16 else "bf16"
    seqs = decoder.PagedSequences(48, 16)
    ids = [seqs.add(), seqs.add()]
    w = [R.weights(c.cpu().numpy(), num(s), num(m), group, name) for c, s, m in (decoder.quantise_weights4(x, group, dtype) for x in raw)]
    norm = num(layer.feed_forward_norm)
    for counts in ([150, 31], [1, 1], [0, 1], [20, 1]):
        step = seqs.extend(ids, counts)
        x = torch.randn(sum(counts), hidden, device=DEV).to(dtype)
        seen = {}
        attend = layer.attention.forward

        def noted(h, st):
            seen["h"], seen["a"] = h, attend(h, st)
            return seen["a"]

        layer.attention.forward = noted
        y = layer.forward(x, step)
        layer.attention.forward = attend
        torch.cuda.synchronize()
        assert ifq.ifq_device_status() == ifq.IFQ_OK
        want, _ = R.rms_norm(num(x), None, num(layer.attention_norm), float(np.float32(1e-5)), name)
        small = 2.0 ** -25 if name == "f16" else 2.0 ** -134
        assert (np.abs(num(seen["h"]) - want) <= np.abs(want) * (R.half_step(name) + 2.0 ** -18) + small).all()
        # the second half, from what attention gave: each stage once more by itself, and the references of those
        h, total = decoder.rms_norm(seen["a"], layer.feed_forward_norm, layer.eps, x)
        want, s = R.rms_norm(num(seen["a"]), num(x), norm, float(np.float32(1e-5)), name)
        assert np.array_equal(num(total), s)
        assert (np.abs(num(h) - want) <= np.abs(want) * (R.half_step(name) + 2.0 ** -18) + small).all()
        mid = layer.feed_forward.first.gate(h, act)
        want, tol = R.gated(num(h), w[0], w[1], act, name)
        assert (np.abs(num(mid) - want) <= tol + small).all()
        want, tol = R.products(num(mid), w[2])
        want = want + s
        assert (np.abs(num(y) - want) <= tol + (2.0 ** -24 + R.half_step(name)) * (np.abs(want) + tol)).all()


def test_a_head_and_its_scores():
    hidden, vocab = 264, 5003
    head = decoder.Head(torch.randn(vocab, hidden, device=DEV), torch.ones(hidden, device=DEV), 64)
    for rows in (1, 5, 40):
        x = torch.randn(rows, hidden, device=DEV).bfloat16()
        logits = head.logits(x)
        tokens = torch.randint(0, vocab, (rows,), device=DEV)
        s = decoder.token_scores(logits, tokens, top=5, temperature=0.8)
        want = R.scores(num(logits), tokens.tolist(), float(np.float32(1 / 0.8)), 5)
        tol = R.scores_tolerance(num(logits), 1 / 0.8)
        assert np.array_equal(num(s.top_ids), want["top_ids"])
        assert (np.abs(num(s.logprobs) - want["logprobs"]) <= tol).all() and (np.abs(num(s.lse) - want["lse"]) <= tol).all()
        assert (np.abs(num(s.entropy) - want["entropy"]) <= 16 * tol).all()
        assert (np.abs(num(s.top_logprobs) - want["top_logprobs"]) <= tol[:, None]).all()


def test_answering_in_a_graph_and_on_two_streams():
    """Greedy steps of two batches: one after the other, at once on two streams, and a captured step replayed after others."""
    layer, _ = layer_of(256, 512, 4, 2, 64, torch.bfloat16, 128)
    head = decoder.Head(torch.randn(1000, 256, device=DEV) * 0.1, torch.ones(256, device=DEV))
    table = torch.randn(1000, 256, device=DEV).bfloat16()
    seqs = decoder.PagedSequences(48, 16)
    batches = [[seqs.add() for _ in range(3)] for _ in range(2)]
    prompts = [[seqs.extend(b, c) for c in ([40, 3, 17], [1, 1, 1], [1, 1, 1])] for b in batches]
    start = [torch.randint(0, 1000, (60,), device=DEV) for _ in range(2)]

    def step(tokens, st):
        y = layer.forward(table[tokens], st)
        last = y[(st.starts[1:] - 1).long()]
        s = decoder.token_scores(head.logits(last), top=2)
        return s.top_ids[:, 0], s

    def answer(i):
        tokens, out = start[i], []
        for st in prompts[i]:
            tokens, s = step(tokens, st)
            out += [tokens, s.lse, s.entropy, s.top_ids, s.top_logprobs]
        return out

    want = [[t.clone() for t in answer(i)] for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [None, None]
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = answer(i)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    tokens = want[0][5]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, s = step(tokens, prompts[0][2])
    answer(1)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0][10]) and torch.equal(s.lse, want[0][11])
    assert ifq.ifq_device_status() == ifq.IFQ_OK
