"""Products in e4m3 with a scale per block of 128, and the quantiser of their activations.

Codes and scales are exact.  The product's tolerance: a sum of K products in single precision errs by at most
2 (128 + blocks) 2^-24 of the sum of the terms' absolute values (128 terms within a block, then the blocks; twice for
sums that truncate), and the result's own rounding comes on top."""
import numpy as np
import pytest
import torch

import lm_reference as R
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"f16": (ifq.IFQ_F16, torch.float16, 2.0 ** -11), "bf16": (ifq.IFQ_BF16, torch.bfloat16, 2.0 ** -8),
         "f32": (ifq.IFQ_F32, torch.float32, 2.0 ** -23)}


@pytest.mark.parametrize("m,k,dtype,pad", [(1, 128, "bf16", 0), (1, 16, "f16", 0), (5, 144, "bf16", 8), (33, 1040, "f16", 24),
                                           (130, 400, "bf16", 0), (700, 256, "f16", 0)])
def test_quantised_activations_are_exact(m, k, dtype, pad):
    rng = np.random.default_rng(m + k)
    x = rng.normal(size=(m, k + pad)).astype(np.float32) * np.exp(rng.normal(0, 2, (m, 1))).astype(np.float32)
    x[m // 2, : min(k, 128)] = 0
    code, dt, _ = TYPES[dtype]
    xd = torch.from_numpy(x).to(DEV).to(dt)
    q = torch.full((m, k), 0x7F, dtype=torch.uint8, device=DEV)
    s = torch.full((-(-k // 128), m), -1.0, device=DEV)
    ifq.ifq_fp8_quantize(ifq.fp8_desc(m, 8, k, code, x_stride=k + pad), xd, q, s)
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
    qw, sw = R.fp8_quantise(xd.float().cpu().numpy()[:, :k])
    tab = R.e4m3_table()
    assert np.array_equal(s.cpu().numpy(), sw)
    assert np.array_equal(tab[q.cpu().numpy()], tab[qw])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quantised_activations_are_exact_near_middles_of_codes(dtype):
    # every half or bfloat16 of a few binades against largest values around 448 2^e, where quotients meet the middles
    code, dt, _ = TYPES[dtype]
    bits = {"bf16": 7, "f16": 10}[dtype]
    mant = np.concatenate([2.0 ** e * (1 + np.arange(2 ** bits) / 2 ** bits) for e in range(-8, 9)]).astype(np.float32)
    rows = []
    for top in (448, 449, 450, 452, 455, 440, 512, 511, 480, 300, 257, 256):
        t = np.concatenate([mant[mant <= top], np.zeros(-len(mant[mant <= top]) % 112, np.float32)]).reshape(-1, 112)
        t = np.concatenate([t * np.where(np.arange(112) % 3 == 0, -1, 1), np.full((len(t), 16), top)], 1)
        rows += [t * 2.0 ** e for e in (0, -7, 5)]
    x = np.concatenate(rows).astype(np.float32)
    m = len(x)
    xd = torch.from_numpy(x).to(DEV).to(dt)
    q, s = torch.empty(m, 128, dtype=torch.uint8, device=DEV), torch.empty(1, m, device=DEV)
    ifq.ifq_fp8_quantize(ifq.fp8_desc(m, 8, 128, code), xd, q, s)
    qw, sw = R.fp8_quantise(xd.float().cpu().numpy())
    tab = R.e4m3_table()
    assert np.array_equal(s.cpu().numpy(), sw)
    assert np.array_equal(tab[q.cpu().numpy()], tab[qw])


def test_quantiser_says_what_is_not_finite():
    x = torch.ones(3, 256, device=DEV).bfloat16()
    x[0, 3], x[1, 200], x[2, 255] = float("nan"), float("inf"), -float("inf")
    q, s = torch.empty(3, 256, dtype=torch.uint8, device=DEV), torch.empty(2, 3, device=DEV)
    ifq.ifq_fp8_quantize(ifq.fp8_desc(3, 8, 256), x, q, s)
    s = s.cpu()
    assert torch.isnan(s[0, 0]) and torch.isinf(s[1, 1]) and torch.isinf(s[1, 2])
    assert torch.isfinite(s[[1, 0, 0], [0, 1, 2]]).all()


def _operands(rng, m, n, k):
    tab = R.e4m3_table()
    fin = np.flatnonzero(np.isfinite(tab))
    # codes as a quantiser leaves them: magnitudes spread over the format, largest near the top
    xq = fin[rng.integers(0, len(fin), (m, k))].astype(np.uint8)
    wq = fin[rng.integers(0, len(fin), (n, k))].astype(np.uint8)
    kb = -(-k // 128)
    xs = np.exp(rng.normal(-5, 1, (kb, m))).astype(np.float32)
    ws = np.exp(rng.normal(-5, 1, (-(-n // 128), kb))).astype(np.float32)
    return xq, xs, wq, ws


def _matmul(xq, xs, wq, ws, out_dtype, pad=0, stream=None):
    m, k = xq.shape
    n = wq.shape[0]
    code, dt, u = TYPES[out_dtype]
    out = torch.full((m, n + pad), 7.0, dtype=dt, device=DEV)
    d = ifq.fp8_desc(m, n, k, ifq.IFQ_BF16, code, out_stride=n + pad)
    size = ifq.ifq_fp8_workspace_bytes(d)
    w = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    args = [torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for a in (xq, xs, wq, ws)]
    torch.cuda.synchronize()
    ifq.ifq_fp8_matmul(d, *args, out, w, size, stream=stream)
    torch.cuda.synchronize()
    first = out.clone()
    ifq.ifq_fp8_matmul(d, *args, out, w, size, stream=stream)
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
    assert torch.equal(out.view(torch.uint8), first.view(torch.uint8))
    assert (out[:, n:] == 7).all()
    return out[:, :n].double().cpu().numpy(), u


SHAPES = [
    # m, n, k, out, pad
    (1, 8, 16, "bf16", 0), (1, 128, 128, "f32", 0), (1, 1000, 1152, "f16", 0), (2, 130, 4112, "bf16", 2),
    (7, 256, 256, "f32", 1), (16, 384, 512, "bf16", 0), (17, 129, 272, "f16", 0), (31, 1, 144, "f32", 0),
    (33, 513, 1040, "bf16", 3), (64, 512, 2048, "f16", 0), (65, 255, 384, "f32", 5), (100, 640, 896, "bf16", 0),
    (127, 257, 160, "f16", 0), (128, 128, 128, "bf16", 0), (129, 384, 640, "f32", 0), (200, 1000, 528, "bf16", 8),
    (256, 256, 1024, "f16", 0), (300, 777, 2064, "bf16", 7), (513, 300, 400, "f32", 0), (1025, 520, 256, "bf16", 0),
]


@pytest.mark.parametrize("m,n,k,out,pad", SHAPES)
def test_product_equals_its_definition(m, n, k, out, pad):
    rng = np.random.default_rng(m * 3 + n)
    xq, xs, wq, ws = _operands(rng, m, n, k)
    got, u = _matmul(xq, xs, wq, ws, out, pad)
    want, mag = R.fp8_matmul(xq, xs, wq, ws)
    tol = u * np.abs(want) + 2 * (128 + xs.shape[0]) * 2.0 ** -24 * mag
    far = np.abs(got - want) - tol
    assert (far <= 0).all(), (far.max(), np.argwhere(far > 0)[:4])


@pytest.mark.parametrize("m,n,k,out,pad", [(2500, 2041, 272, "f32", 3), (2305, 2177, 528, "bf16", 7), (130, 19600, 400, "f16", 0),
                                           (5000, 4000, 144, "bf16", 0)])
def test_large_product_equals_its_definition(m, n, k, out, pad):
    test_product_equals_its_definition(m, n, k, out, pad)


@pytest.mark.parametrize("m,n,k", [(3, 200, 400), (70, 130, 256), (260, 256, 384)])
def test_a_row_that_is_not_finite_stays_by_itself(m, n, k):
    rng = np.random.default_rng(m)
    xq, xs, wq, ws = _operands(rng, m, n, k)
    clean, _ = _matmul(xq, xs, wq, ws, "f32")
    x2, s2 = xq.copy(), xs.copy()
    x2[1, 130] = 0x7F
    s2[0, 2] = np.inf
    got, _ = _matmul(x2, s2, wq, ws, "f32")
    assert np.isnan(got[1]).all() and not np.isfinite(got[2]).any()
    keep = np.arange(m) > 2
    assert np.array_equal(got[keep], clean[keep]) and np.array_equal(got[0], clean[0])


def test_zero_blocks_and_no_rows():
    rng = np.random.default_rng(0)
    xq, xs, wq, ws = _operands(rng, 40, 256, 384)
    xs[1], xq[:, 128:256] = 0, 0
    got, u = _matmul(xq, xs, wq, ws, "f32")
    want, mag = R.fp8_matmul(xq, xs, wq, ws)
    assert (np.abs(got - want) <= 2 * 131 * 2.0 ** -24 * mag + u * np.abs(want)).all()
    out = torch.full((1, 256), 3.0, device=DEV)
    d = ifq.fp8_desc(0, 256, 384, out_dtype=ifq.IFQ_F32)
    one = torch.zeros(16, dtype=torch.uint8, device=DEV)
    ifq.ifq_fp8_matmul(d, one, one, one, one, out, one, 16)
    ifq.ifq_fp8_quantize(d, one, one, one)
    torch.cuda.synchronize()
    assert (out == 3).all()


def test_product_on_another_stream():
    rng = np.random.default_rng(1)
    for m in (4, 150):
        ops = _operands(rng, m, 300, 512)
        a, _ = _matmul(*ops, "bf16")
        b, _ = _matmul(*ops, "bf16", stream=torch.cuda.Stream())
        assert np.array_equal(a, b)
