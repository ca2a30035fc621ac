"""Attention with as many key heads as a cache may have."""
import numpy as np
import pytest
import torch

import test_gpu_kv4 as base
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 33])
def test_65536_key_heads(n):
    """Eight heads' cache and queries, repeated: every copy gives the same, and the first what its definition says."""
    rng = np.random.default_rng(31)
    hk, D, page, times = 8, 64, 16, 8192
    lens, starts, table, cache, q = base._setup(rng, [40], [n], hk, hk, D, page)
    big = base._dev(cache).repeat(1, times, 1, 1)
    qd = base._dev(q.reshape(n, -1), torch.bfloat16)
    d = ifq.kv4_attention_desc(ifq.kv4_cache(big.shape[0], page, hk * times, D), 1, n, n, table.shape[1], hk * times,
                               ifq.IFQ_BF16, D ** -0.5)
    out = torch.full((n, times, hk * D), 5.0, dtype=torch.bfloat16, device=base.DEV)
    size = ifq.ifq_kv4_attention_workspace_bytes(d)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device=base.DEV)
    ifq.ifq_kv4_attention(d, qd.repeat(1, times), big, base._dev(table), base._dev(lens), base._dev(starts), out, None, ws, size)
    assert base._status() == ifq.IFQ_OK
    assert (out == out[:, :1]).all()
    u = base.TYPES["bf16"][2]
    got = (out[:, 0].double().cpu().numpy().reshape(n, hk, D), None, qd.double().cpu().numpy().reshape(n, hk, D), D ** -0.5, u, n > 32)
    base._check(got, lens, starts, table, cache, hk, page, lse=False)
