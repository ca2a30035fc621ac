"""Products with 4-bit weights whose codes go through rings of shared memory that hold few blocks: whole numbers must come out
exactly, call after call, while another stream's copies fill the memory, so that the rings' copies land in any order."""
import numpy as np
import pytest
import torch

import layer_reference as R
from paper_1911_08076_gb300 import ifq
from test_gpu_w4 import TYPES, activations, draw, to_dev

pytestmark = pytest.mark.gpu

DEV = "cuda"


def exact_products(m, n, k, group, dtype, out, distinct=637, calls=12):
    """n rows of w, of which `distinct` follow each other again and again (a number that no tile's rows divide)."""
    rng = np.random.default_rng([m, n, k, group])
    distinct = min(distinct, n)
    w = ifq.w4_weights(n, k, group, TYPES[dtype][0])
    codes, scales, mins, values = draw(rng, distinct, k, group, dtype, True)
    at = torch.arange(n, device=DEV) % distinct
    packed = torch.empty(ifq.ifq_w4_bytes(w), dtype=torch.uint8, device=DEV)
    ifq.ifq_w4_pack(w, torch.from_numpy(codes).to(DEV)[at], to_dev(scales, dtype)[at], to_dev(mins, dtype)[at], packed)
    x = activations(rng, m, k, dtype, True)
    want = torch.from_numpy(R.round_to(x @ values.T, out)).to(DEV)[:, at].to(TYPES[out][1])
    xd, busy = to_dev(x, dtype), torch.cuda.Stream()
    big, to = torch.zeros(1 << 26, device=DEV), torch.empty(1 << 26, device=DEV)
    got = [torch.full((m, n), 7.0, device=DEV, dtype=TYPES[out][1]) for _ in range(calls)]
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        with torch.cuda.stream(busy):
            if i % 3:
                to.copy_(big)
        ifq.ifq_w4_matmul(ifq.w4_desc(w, m, TYPES[out][0]), xd, packed, y)
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
    for y in got:
        assert torch.equal(y, want)


# Two full turns of tiles on 152 SMs.  Blocks of 128 columns that three (m <= 8) or two warps take in turn, from two to nine stages
# each: numbers of blocks that the turns divide, and that they do not.  (x of 8 x 10240 leaves no room for a ring.)
@pytest.mark.parametrize("m,k,group,dtype", [(8, 8192, 128, "bf16"), (8, 8192, 32, "f16"), (8, 10240, 128, "bf16"), (12, 6144, 64, "bf16"),
                                             (16, 5000, 32, "f16"), (5, 12296, 128, "bf16"), (5, 4232, 128, "bf16"), (16, 2056, 32, "bf16"),
                                             (8, 4096, 64, "bf16"), (6, 328, 64, "f16"), (9, 4096, 128, "bf16"), (7, 136, 32, "bf16"),
                                             (16, 8, 128, "f16")])
def test_many_rows_of_weights(m, k, group, dtype):
    exact_products(m, 38859, k, group, dtype, "f32")


@pytest.mark.parametrize("m,k,group,dtype,act", [(8, 4096, 64, "bf16", "silu"), (6, 1032, 32, "f16", "gelu_tanh"), (13, 4232, 128, "bf16", "gelu")])
def test_many_rows_of_a_gated_pair(m, k, group, dtype, act):
    n, distinct = 19450, 331
    rng = np.random.default_rng([m, k, group])
    w = ifq.w4_weights(n, k, group, TYPES[dtype][0], True)
    codes, scales, mins, values = draw(rng, 2 * distinct, k, group, dtype, False)
    at = torch.arange(n, device=DEV) % distinct
    at = torch.cat([at, at + distinct])
    packed = torch.empty(ifq.ifq_w4_bytes(w), dtype=torch.uint8, device=DEV)
    ifq.ifq_w4_pack(w, torch.from_numpy(codes).to(DEV)[at], to_dev(scales, dtype)[at], to_dev(mins, dtype)[at], packed)
    x = activations(rng, m, k, dtype, False)
    want, tol = R.gated(x, values[:distinct], values[distinct:], act, dtype)
    if dtype == "f16":
        tol = tol + 2.0 ** -25     # half of the smallest half
    first = None
    for _ in range(4):
        out = torch.full((m, n), 7.0, device=DEV, dtype=TYPES[dtype][1])
        ifq.ifq_w4_gated(ifq.w4_desc(w, m, TYPES[dtype][0], R.ACTS[act]), to_dev(x, dtype), packed, out)
        got = out.double().cpu().numpy()
        idx = np.arange(n) % distinct
        assert (np.abs(got - want[:, idx]) <= tol[:, idx]).all()
        assert first is None or torch.equal(out, first)
        first = out
    assert ifq.ifq_device_status() == ifq.IFQ_OK


# Floats whose k is split, in parts of more than one chain: the fewest slots for codes beside the sums (two to six).  And the sizes
# with seven and more.
@pytest.mark.parametrize("m,n,k,group,out", [(128, 130, 16384, 128, "f32"), (128, 130, 16384, 64, "f32"), (128, 100, 16392, 32, "f32"),
                                             (96, 130, 16384, 64, "f32"), (96, 250, 16384, 32, "f32"), (96, 130, 12296, 128, "f32"),
                                             (80, 130, 16384, 128, "f32"), (112, 130, 16384, 64, "f32"), (120, 130, 13000, 128, "bf16"),
                                             (128, 4000, 4096, 128, "f32"), (600, 2000, 9216, 128, "bf16"), (700, 2000, 4096, 64, "f32")])
def test_many_rows_of_x(m, n, k, group, out):
    exact_products(m, n, k, group, "bf16", out)
