"""A quantised decoder layer: attention with e4m3 projections over a 4-bit paged cache, a gated feed-forward block with
4-bit weights, the norms between them, and the scores of its answers.

PagedSequences keeps, on the host, which pages belong to which sequence and gives a step's index tensors;
DecoderAttention holds the quantised weights and the cache, and runs a step (a batch of sequences with
one or several new tokens each) as six calls on the current stream:

    quantise x, x Wqkv^T, rotate + quantise + append, attend, quantise the context, context Wo^T

FeedForward is act(x Wg^T) * (x Wu^T) and the product with Wd, DecoderLayer puts a norm before each block and adds its result
to the stream, and Head turns the stream into logits and token_scores those into log probabilities and the likeliest
tokens.  All compute is in libifq.so.
"""
from __future__ import annotations

import math
from typing import List, NamedTuple, Optional, Sequence

import numpy as np
import torch

from . import ifq

TYPES = {torch.float16: ifq.IFQ_F16, torch.bfloat16: ifq.IFQ_BF16}


def quantise_weights(w: torch.Tensor):
    """Weights [n][k] (k a multiple of 16) to e4m3 with a scale per 128 x 128 block, once: (codes, scales)."""
    n, k = w.shape
    nb, kb = -(-n // 128), -(-k // 128)
    padded = torch.zeros(nb * 128, kb * 128, dtype=torch.float32, device=w.device)
    padded[:n, :k] = w.float()
    blocks = padded.view(nb, 128, kb, 128)
    scales = (blocks.abs().amax((1, 3)) / 448.0).clamp_min(1e-30).contiguous()
    codes = (blocks / scales[:, None, :, None]).view(nb * 128, kb * 128)[:n, :k].contiguous().to(torch.float8_e4m3fn)
    return codes, scales


def rotation_tables(positions: int, rot_dim: int, base: float = 10000.0, device="cuda"):
    """cos and sin of position * base^(-2 i / rot_dim), float [positions][rot_dim / 2]."""
    freq = base ** (-torch.arange(0, rot_dim, 2, device=device, dtype=torch.float64) / rot_dim)
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * freq
    return angle.cos().float().contiguous(), angle.sin().float().contiguous()


class Step:
    """Index tensors of one step (device), the sizes that choose the kernels, and the pool that its pages are of (host)."""

    def __init__(self, positions, slots, lens, starts, table, max_q, max_len, pages=None, page_size=None):
        self.positions, self.slots, self.lens, self.starts, self.table = positions, slots, lens, starts, table
        self.max_q, self.max_len = max_q, max_len
        self.pages, self.page_size = pages, page_size


class PagedSequences:
    """Page bookkeeping of a batch of sequences over `pages` pages of `page_size` tokens."""

    def __init__(self, pages: int, page_size: int, device="cuda"):
        self.count, self.page_size, self.device = pages, page_size, torch.device(device)
        self.free: List[int] = list(range(pages - 1, -1, -1))
        self.pages: List[List[int]] = []
        self.length: List[int] = []

    def add(self) -> int:
        """A new, empty sequence; its number."""
        self.pages.append([])
        self.length.append(0)
        return len(self.length) - 1

    def release(self, seq: int):
        """Give a sequence's pages back; it is empty then."""
        self.free.extend(reversed(self.pages[seq]))
        self.pages[seq], self.length[seq] = [], 0

    def extend(self, seqs: Sequence[int], counts: Sequence[int]) -> Step:
        """Room for counts[i] new tokens of sequence seqs[i] (the tokens in this order in the step's rows)."""
        need = [-(-(self.length[s] + n) // self.page_size) - len(self.pages[s]) for s, n in zip(seqs, counts)]
        if len(set(seqs)) != len(seqs) or any(n < 0 for n in counts):
            raise ValueError("a sequence comes once in a step, with no fewer than 0 tokens")
        if sum(need) > len(self.free):
            raise MemoryError(f"{sum(need)} pages are needed and {len(self.free)} are free")
        positions, slots = [], []
        for s, n, more in zip(seqs, counts, need):
            self.pages[s].extend(self.free.pop() for _ in range(more))
            p = np.arange(self.length[s], self.length[s] + n)
            positions.append(p)
            slots.append(np.asarray(self.pages[s], np.int64)[p // self.page_size] * self.page_size + p % self.page_size
                         if n else p)
            self.length[s] += n
        table = np.zeros((len(seqs), max([1] + [len(self.pages[s]) for s in seqs])), np.int32)
        for i, s in enumerate(seqs):
            table[i, :len(self.pages[s])] = self.pages[s]
        lens = np.array([self.length[s] for s in seqs], np.int32)
        dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, t)).to(self.device)   # noqa: E731
        cat = lambda a, t: dev(np.concatenate(a) if a else np.zeros(0), t)               # noqa: E731
        return Step(cat(positions, np.int32), cat(slots, np.int64), dev(lens, np.int32),
                    dev(np.concatenate([[0], np.cumsum(counts)]), np.int32), dev(table, np.int32),
                    max([0] + list(counts)), int(lens.max(initial=0)), self.count, self.page_size)


class DecoderAttention:
    """x -> attention block output.  w_qkv [(q_heads + 2 kv_heads) * head_dim][hidden], w_out [hidden][q_heads * head_dim]."""

    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, q_heads: int, kv_heads: int, head_dim: int, pages: int,
                 page_size: int = 64, max_positions: int = 4096, dtype: torch.dtype = torch.bfloat16,
                 rot_dim: Optional[int] = None, rope: int = ifq.IFQ_ROPE_HALVES, rope_base: float = 10000.0,
                 window: int = 0, sinks: int = 0):
        dev = w_qkv.device
        self.hidden, self.q_heads, self.kv_heads, self.head_dim = w_qkv.shape[1], q_heads, kv_heads, head_dim
        if tuple(w_qkv.shape) != ((q_heads + 2 * kv_heads) * head_dim, self.hidden) or \
                tuple(w_out.shape) != (self.hidden, q_heads * head_dim):
            raise ValueError("w_qkv is [(q_heads + 2 kv_heads) * head_dim][hidden], w_out [hidden][q_heads * head_dim]")
        self.dtype, self.code, self.rope, self.window, self.sinks = dtype, TYPES[dtype], rope, window, sinks
        self.rot_dim = head_dim if rot_dim is None else rot_dim
        self.w_qkv, self.s_qkv = quantise_weights(w_qkv)
        self.w_out, self.s_out = quantise_weights(w_out)
        self.cos, self.sin = rotation_tables(max_positions, self.rot_dim, rope_base, dev)
        self.pool = ifq.kv4_cache(pages, page_size, kv_heads, head_dim)
        self.cache = torch.zeros(ifq.ifq_kv4_cache_bytes(self.pool), dtype=torch.uint8, device=dev)

    def _room(self, size):
        return torch.empty(max(size, 1), dtype=torch.uint8, device=self.cache.device)

    def _product(self, x, w, scales):
        rows, k = x.shape
        d = ifq.fp8_desc(rows, w.shape[0], k, self.code, self.code)
        out = torch.empty(rows, w.shape[0], dtype=self.dtype, device=x.device)
        codes = torch.empty(rows, k, dtype=torch.float8_e4m3fn, device=x.device)
        xs = torch.empty(-(-k // 128), rows, dtype=torch.float32, device=x.device)
        size = ifq.ifq_fp8_workspace_bytes(d)
        ifq.ifq_fp8_quantize(d, x, codes, xs)
        ifq.ifq_fp8_matmul(d, codes, xs, w, scales, out, self._room(size), size)
        return out

    def forward(self, x: torch.Tensor, step: Step) -> torch.Tensor:
        """x [tokens][hidden], the tokens of `step` in order -> [tokens][hidden].  ValueError where a sequence runs past
        max_positions, or the step's pages are not those of the cache."""
        if x.dtype != self.dtype or not x.is_contiguous() or x.shape != (step.positions.numel(), self.hidden):
            raise ValueError("x is a dense [tokens][hidden] tensor of the block's dtype, a row a token of the step")
        # (the calls would skip such tokens, and say so in the device's status alone)
        if self.rope != ifq.IFQ_ROPE_NONE and step.max_len > self.cos.shape[0]:
            raise ValueError(f"a sequence of {step.max_len} tokens runs past the {self.cos.shape[0]} positions of the tables")
        if step.page_size not in (None, self.pool.page_size) or (step.pages or 0) > self.pool.pages:
            raise ValueError(f"the step's pages ({step.pages} of {step.page_size} tokens) are not the cache's "
                             f"({self.pool.pages} of {self.pool.page_size})")
        rows, hq, hk, d = x.shape[0], self.q_heads, self.kv_heads, self.head_dim
        wide = (hq + 2 * hk) * d
        # Every step's buffers are its own, from torch's allocator for the current stream (or the graph being captured), so
        # steps on several streams and replays of captured ones do not meet.  self.qkv, self.q and self.context are the last
        # step's.
        qkv = self.qkv = self._product(x, self.w_qkv, self.s_qkv)
        q = self.q = torch.empty(rows, hq * d, dtype=self.dtype, device=x.device)
        a = ifq.kv4_append_desc(self.pool, rows, hq, self.code, self.rope, self.rot_dim, self.cos.shape[0],
                                q_stride=wide, k_stride=wide, v_stride=wide)
        ifq.ifq_kv4_append(a, qkv, qkv[:, hq * d:], qkv[:, (hq + hk) * d:], self.cos, self.sin, step.positions, step.slots,
                           q, self.cache)
        context = self.context = torch.empty(rows, hq * d, dtype=self.dtype, device=x.device)
        t = ifq.kv4_attention_desc(self.pool, step.lens.numel(), rows, step.max_q, step.table.shape[1], hq, self.code,
                                   1.0 / math.sqrt(d), self.window, self.sinks, max_len=step.max_len)
        size = ifq.ifq_kv4_attention_workspace_bytes(t)
        ifq.ifq_kv4_attention(t, q, self.cache, step.table, step.lens, step.starts, context, None, self._room(size), size)
        return self._product(context, self.w_out, self.s_out)


def _check_devices(first, *others):
    """ValueError unless all tensors (or None) are on one device, the current one: the calls take their addresses."""
    device = first.device
    if any(t is not None and t.device != device for t in others) or \
            (device.type == "cuda" and device.index != torch.cuda.current_device()):
        raise ValueError("all tensors are on one device, the current one")


ACTS = {"silu": ifq.IFQ_ACT_SILU, "gelu": ifq.IFQ_ACT_GELU, "gelu_tanh": ifq.IFQ_ACT_GELU_TANH}


def quantise_weights4(w: torch.Tensor, group: int = 128, dtype: torch.dtype = torch.bfloat16):
    """Weights [n][k] (k a multiple of 8) to 4 bits with a scale and a minimum of `dtype` per row and group of columns, once:
    (codes [n][k / 2], scales [n][groups], mins [n][groups])."""
    n, k = w.shape
    groups = -(-k // group)
    pad = groups * group - k
    f = w.float()
    low = torch.nn.functional.pad(f, (0, pad), value=math.inf).view(n, groups, group).amin(-1)
    high = torch.nn.functional.pad(f, (0, pad), value=-math.inf).view(n, groups, group).amax(-1)
    scales, mins = ((high - low) / 15.0).to(dtype), low.to(dtype)
    s, m = (t.float().repeat_interleave(group, 1)[:, :k] for t in (scales, mins))
    codes = torch.where(s > 0, ((f - m) / s).round().clamp(0, 15), torch.zeros_like(f)).to(torch.uint8)
    return codes[:, 0::2] | (codes[:, 1::2] << 4), scales, mins


class Weights4:
    """A matrix [n][k] in 4 bits, or a gated pair of them (the gate's, the other's), packed for the products."""

    def __init__(self, *matrices: torch.Tensor, group: int = 128, dtype: torch.dtype = torch.bfloat16):
        if len(matrices) not in (1, 2) or any(m.shape != matrices[0].shape for m in matrices):
            raise ValueError("one matrix [n][k], or a gated pair of the same shape")
        self.n, self.k = matrices[0].shape
        self.dtype, self.gated = dtype, len(matrices) == 2
        self.desc = ifq.w4_weights(self.n, self.k, group, TYPES[dtype], self.gated)
        size = ifq.ifq_w4_bytes(self.desc)
        parts = [quantise_weights4(m, group, dtype) for m in matrices]
        codes, scales, mins = (torch.cat(p).contiguous() for p in zip(*parts))
        _check_devices(codes)
        self.packed = torch.empty(size, dtype=torch.uint8, device=codes.device)
        ifq.ifq_w4_pack(self.desc, codes, scales, mins, self.packed)

    def _rows(self, x):
        # (rows that share their storage, as an expanded tensor's: a stride of 0 would mean dense)
        if x.dim() != 2 or x.dtype != self.dtype or x.shape[1] != self.k or x.stride(1) != 1 or \
                (x.shape[0] > 1 and (x.stride(0) % 8 or x.stride(0) < self.k)):
            raise ValueError(f"x is a [rows][{self.k}] tensor of {self.dtype}, rows a multiple of 8 elements apart and of its own")
        _check_devices(x, self.packed)
        return x.shape[0], x.stride(0) if x.shape[0] > 1 else 0

    def matmul(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
        """x w^T (+ residual), x [rows][k] -> [rows][n] of out_dtype (the weights' where none is given)."""
        rows, stride = self._rows(x)
        out_dtype = out_dtype or self.dtype
        if residual is not None and (residual.shape != (rows, self.n) or residual.dtype != out_dtype or not residual.is_contiguous()):
            raise ValueError("residual is a dense tensor of the result's shape and type")
        if residual is not None:
            _check_devices(x, residual)
        out = torch.empty(rows, self.n, dtype=out_dtype, device=x.device)
        d = ifq.w4_desc(self.desc, rows, ifq.IFQ_F32 if out_dtype == torch.float32 else TYPES[out_dtype], 0, stride)
        ifq.ifq_w4_matmul(d, x, self.packed, out, residual)
        return out

    def gate(self, x: torch.Tensor, act: str = "silu") -> torch.Tensor:
        """act(x wg^T) * (x wu^T) of a gated pair."""
        rows, stride = self._rows(x)
        out = torch.empty(rows, self.n, dtype=self.dtype, device=x.device)
        ifq.ifq_w4_gated(ifq.w4_desc(self.desc, rows, TYPES[self.dtype], ACTS[act], stride), x, self.packed, out)
        return out


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: Optional[torch.Tensor] = None):
    """Norm of the rows of x [rows][dim]; with a residual (norm of x + residual, x + residual)."""
    if x.dim() != 2 or not x.is_contiguous() or weight.shape != x.shape[1:] or weight.dtype != x.dtype or not weight.is_contiguous() or \
            (residual is not None and (residual.shape != x.shape or residual.dtype != x.dtype or not residual.is_contiguous())):
        raise ValueError("x and residual are dense [rows][dim] tensors, weight [dim], all of one type")
    _check_devices(x, weight, residual)
    out, total = torch.empty_like(x), None if residual is None else torch.empty_like(x)
    ifq.ifq_rms_norm(ifq.norm_desc(x.shape[0], x.shape[1], TYPES[x.dtype], eps), x, residual, weight, total, out)
    return out if residual is None else (out, total)


class FeedForward:
    """x -> act(x w_gate^T) * (x w_up^T), times w_down^T.  w_gate, w_up [inner][hidden], w_down [hidden][inner]."""

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, act: str = "silu", group: int = 128,
                 dtype: torch.dtype = torch.bfloat16):
        if w_down.shape != w_gate.shape[::-1]:
            raise ValueError("w_gate and w_up are [inner][hidden], w_down [hidden][inner]")
        self.act = act
        self.first, self.second = Weights4(w_gate, w_up, group=group, dtype=dtype), Weights4(w_down, group=group, dtype=dtype)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        return self.second.matmul(self.first.gate(x, self.act), residual)


class DecoderLayer:
    """stream -> stream: stream + attention(norm(stream)), then that + feed_forward(norm(that))."""

    def __init__(self, attention: DecoderAttention, feed_forward: FeedForward, attention_norm: torch.Tensor,
                 feed_forward_norm: torch.Tensor, eps: float = 1e-5):
        self.attention, self.feed_forward, self.eps = attention, feed_forward, eps
        self.attention_norm, self.feed_forward_norm = (w.to(attention.dtype).contiguous() for w in (attention_norm, feed_forward_norm))

    def forward(self, x: torch.Tensor, step: Step) -> torch.Tensor:
        a = self.attention.forward(rms_norm(x, self.attention_norm, self.eps), step)
        h, x = rms_norm(a, self.feed_forward_norm, self.eps, x)
        return self.feed_forward.forward(h, x)


class Scores(NamedTuple):
    logprobs: Optional[torch.Tensor]       # of the given tokens (0 where that is negative), [rows]
    lse: torch.Tensor                      # [rows]
    entropy: torch.Tensor                  # [rows]
    top_ids: Optional[torch.Tensor]        # [rows][top], the likeliest first
    top_logprobs: Optional[torch.Tensor]   # [rows][top]


def token_scores(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, temperature: float = 1.0) -> Scores:
    """Scores of rows of logits [rows][vocab] at a temperature; tokens: int64 [rows]."""
    if logits.dim() != 2 or logits.stride(1) != 1 or (logits.shape[0] > 1 and logits.stride(0) < logits.shape[1]) or (tokens is not None and (
            tokens.shape != logits.shape[:1] or tokens.dtype != torch.int64 or not tokens.is_contiguous())):
        raise ValueError("logits are rows [rows][vocab] that share nothing, tokens a dense int64 tensor [rows]")
    _check_devices(logits, tokens)
    rows, vocab = logits.shape
    new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=logits.device)   # noqa: E731
    s = Scores(None if tokens is None else new(rows), new(rows), new(rows), new(rows, top, t=torch.int64) if top else None,
               new(rows, top) if top else None)
    code = ifq.IFQ_F32 if logits.dtype == torch.float32 else TYPES[logits.dtype]
    d = ifq.scores_desc(rows, vocab, code, top, 1.0 / temperature, logits.stride(0) if rows > 1 else 0)
    ifq.ifq_token_scores(d, logits, tokens, *s)
    return s


class Head:
    """The stream's last norm and the product with the vocabulary's rows [vocab][hidden]."""

    def __init__(self, w: torch.Tensor, norm: torch.Tensor, group: int = 128, dtype: torch.dtype = torch.bfloat16, eps: float = 1e-5):
        self.weights, self.norm, self.eps = Weights4(w, group=group, dtype=dtype), norm.to(dtype).contiguous(), eps

    def logits(self, x: torch.Tensor) -> torch.Tensor:
        """float32 [rows][vocab]"""
        return self.weights.matmul(rms_norm(x, self.norm, self.eps), out_dtype=torch.float32)
