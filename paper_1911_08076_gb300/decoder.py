"""The attention block of a quantised decoder layer: e4m3 projections around attention over a 4-bit paged cache.

PagedSequences keeps, on the host, which pages belong to which sequence and gives a step's index tensors;
DecoderAttention holds the quantised weights and the cache, and runs a step (a batch of sequences with
one or several new tokens each) as six calls on the current stream:

    quantise x, x Wqkv^T, rotate + quantise + append, attend, quantise the context, context Wo^T

All compute is in libifq.so.
"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence

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
