"""Products with weights in 4 bits.

Integer weights and activations whose sums stay below 2^24 must come out exactly, whatever the order of the sums, and a
row of x with a single 1 reads the weights back bit by bit.  Real values: see layer_reference."""
import numpy as np
import pytest
import torch

import layer_reference as R
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"f16": (ifq.IFQ_F16, torch.float16), "bf16": (ifq.IFQ_BF16, torch.bfloat16), "f32": (ifq.IFQ_F32, torch.float32)}


def to_dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV).to(TYPES[dtype][1])


def pack(w, codes, scales, mins, dtype):
    packed = torch.full((ifq.ifq_w4_bytes(w) + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    ifq.ifq_w4_pack(w, torch.from_numpy(codes).to(DEV), to_dev(scales, dtype), to_dev(mins, dtype), packed)
    assert (packed[-64:] == 0xA5).all()
    return packed


def draw(rng, rows, k, group, dtype, whole):
    codes = rng.integers(0, 256, (rows, k // 2), np.uint8)
    shape = (rows, -(-k // group))
    if whole:   # values in [-16, 22], all of them exact
        scales, mins = rng.choice([0.5, 1.0, 2.0], shape), rng.integers(-8, -1, shape).astype(np.float64) * 2
        mins = np.where(scales == 2.0, mins, mins / 2)
    else:
        scales = R.round_to(rng.uniform(0.2, 1.0, shape) * 0.02, dtype)
        mins = R.round_to(-7.5 * scales + rng.normal(0, 0.02, shape), dtype)
    return codes, scales, mins, R.weights(codes, scales, mins, group, dtype)


def activations(rng, m, k, dtype, whole):
    return rng.integers(-2, 3, (m, k)).astype(np.float64) if whole else R.round_to(rng.normal(size=(m, k)) *
                                                                                 np.where(rng.random(k) < 0.02, 9, 1), dtype)


def matmul(w, x, packed, dtype, out, residual=None, pads=(0, 0, 0), extra=3):
    """Runs the call on rows with pads of NaN, and checks that what is beside the rows stays as it was."""
    m, k = x.shape
    xd = torch.full((m, k + pads[0]), float("nan"), device=DEV, dtype=TYPES[dtype][1])
    xd[:, :k] = to_dev(x, dtype)
    od = torch.full((m + extra, w.n + pads[1]), 7.0, device=DEV, dtype=TYPES[out][1])
    rd = None
    if residual is not None:
        rd = torch.full((m, w.n + pads[2]), float("nan"), device=DEV, dtype=TYPES[out][1])
        rd[:, :w.n] = to_dev(residual, out)
    d = ifq.w4_desc(w, m, TYPES[out][0], 0, k + pads[0], w.n + pads[1], w.n + pads[2])
    ifq.ifq_w4_matmul(d, xd, packed, od, rd)
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
    assert (od[m:] == 7).all() and (od[:, w.n:] == 7).all()
    return od[:m, :w.n].double().cpu().numpy()


SIZES = [(1, 1, 8), (1, 16, 128), (1, 130, 136), (2, 48, 1024), (3, 257, 264), (5, 64, 4104), (7, 4097, 512), (8, 1000, 640),
         (9, 33, 2056), (15, 300, 384), (16, 512, 1160), (17, 129, 256), (24, 700, 72), (31, 128, 1288), (33, 1025, 520),
         (47, 160, 2560), (64, 96, 8), (65, 640, 328), (100, 2049, 136), (128, 256, 1024), (129, 127, 640), (200, 1152, 264),
         (255, 64, 392), (257, 384, 200), (384, 130, 520), (513, 520, 648), (1000, 260, 136), (4, 40, 33024), (14, 24, 20008),
         (1, 9730, 264), (3, 40007, 128), (6, 12289, 1416), (8, 19600, 8), (12, 10000, 648), (16, 20100, 136)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("group,dtype", [(32, "bf16"), (64, "f16"), (128, "bf16")])
def test_whole_numbers_are_exact(m, n, k, group, dtype):
    rng = np.random.default_rng([m, n, k, group])
    w = ifq.w4_weights(n, k, group, TYPES[dtype][0])
    codes, scales, mins, values = draw(rng, n, k, group, dtype, True)
    packed = pack(w, codes, scales, mins, dtype)
    x = activations(rng, m, k, dtype, True)
    pads = (8 * (m % 3), m % 2, n % 3)
    assert np.array_equal(matmul(w, x, packed, dtype, "f32", pads=pads), x @ values.T)
    res = rng.integers(-99, 99, (m, n)).astype(np.float64)
    got = matmul(w, x, packed, dtype, dtype, res, pads)
    assert np.array_equal(got, R.round_to(x @ values.T + res, dtype))


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("group,dtype,out", [(32, "f16", "f16"), (64, "bf16", "f32"), (128, "bf16", "bf16")])
def test_real_values(m, n, k, group, dtype, out):
    rng = np.random.default_rng([m, n, k, group, 1])
    w = ifq.w4_weights(n, k, group, TYPES[dtype][0])
    codes, scales, mins, values = draw(rng, n, k, group, dtype, False)
    packed = pack(w, codes, scales, mins, dtype)
    x = activations(rng, m, k, dtype, False)
    res = R.round_to(rng.normal(size=(m, n)) * 2, out)
    y, tol = R.products(x, values)
    got = matmul(w, x, packed, dtype, out, res)
    y = y + res
    tol = tol + (2.0 ** -24 + R.half_step(out)) * (np.abs(y) + tol)
    assert (np.abs(got - y) <= tol).all(), np.max(np.abs(got - y) / tol)


@pytest.mark.parametrize("m,n,k", [(5, 200, 12000), (16, 9730, 4096), (40, 300, 16384), (120, 130, 16384), (128, 100, 4096), (100, 2000, 5000),
                                   (300, 300, 16384), (1000, 256, 9216), (1100, 2560, 2048)])
@pytest.mark.parametrize("group", [32, 128])
def test_floats_of_long_sums(m, n, k, group):
    """Sums of one sign, where truncated additions add up: tensor memory adds 64 times 16 products (chains of 1024 columns) at
    most before single precision takes over.  An addition there truncates, by 2^-23 of the sum at most, and on average of
    a growing sum by a quarter of that: 64 / 4 additions' worth for a chain, and for each of the k / 1024 chains' additions,
    k / 128 where a block is one, half a step."""
    rng = np.random.default_rng([m, n, k])
    w = ifq.w4_weights(n, k, group, ifq.IFQ_BF16)
    codes, scales, mins, values = draw(rng, n, k, group, "bf16", False)
    mins = np.abs(mins)
    values = R.weights(codes, scales, mins, group, "bf16")
    packed = pack(w, codes, scales, mins, "bf16")
    x = np.abs(activations(rng, m, k, "bf16", False))
    got, y = matmul(w, x, packed, "bf16", "f32"), x @ values.T
    assert (np.abs(got - y) <= y * (64 + k / 128) * 2.0 ** -24).all(), np.max(np.abs(got - y) / y) * 2 ** 24


@pytest.mark.parametrize("largest", [0.2, 1.0, 300.0])
@pytest.mark.parametrize("m", [8, 200])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_weight_reads_back(m, group, dtype, largest):
    """Rows of x with a single 1: out is the weights, each rounded once from code * scale + min."""
    n, k = 130, 392
    rng = np.random.default_rng(group)
    w = ifq.w4_weights(n, k, group, TYPES[dtype][0])
    codes, scales, mins, values = draw(rng, n, k, group, dtype, False)
    scales[::7], mins[::5] = R.round_to(scales[::7] * 2.0 ** -9, dtype), R.round_to(mins[::5] * 2.0 ** 6, dtype)
    scales[3], mins[4], scales[5] = -scales[3], 0.0, 0.0
    scales[6], scales[8] = R.round_to(2.0 ** (-24 if dtype == 'f16' else -130), dtype), R.round_to(largest, dtype)
    mins[6] = 0.0
    values = R.weights(codes, scales, mins, group, dtype)
    packed = pack(w, codes, scales, mins, dtype)
    for c0 in range(0, k, m):
        cols = np.arange(c0, min(c0 + m, k))
        x = np.zeros((m, k))
        x[np.arange(len(cols)), cols] = 1
        assert np.array_equal(matmul(w, x, packed, dtype, "f32")[:len(cols)], values[:, cols].T)


@pytest.mark.parametrize("m,n,k", [(1, 8, 8), (1, 100, 1032), (4, 65, 264), (8, 1032, 512), (11, 7, 648), (16, 520, 1024),
                                   (19, 129, 264), (40, 600, 136), (64, 64, 1288), (130, 257, 392), (300, 96, 520), (600, 200, 128),
                                   (1, 5003, 392), (7, 10001, 136), (14, 4901, 648)])
@pytest.mark.parametrize("group,dtype,act", [(32, "f16", "gelu_tanh"), (64, "bf16", "gelu"), (128, "bf16", "silu"), (128, "f16", "silu")])
def test_gated(m, n, k, group, dtype, act):
    rng = np.random.default_rng([m, n, k, group, 2])
    w = ifq.w4_weights(n, k, group, TYPES[dtype][0], True)
    codes, scales, mins, values = draw(rng, 2 * n, k, group, dtype, False)
    packed = pack(w, codes, scales, mins, dtype)
    x = activations(rng, m, k, dtype, False)
    pads = (8, 3)
    xd = torch.full((m, k + pads[0]), float("nan"), device=DEV, dtype=TYPES[dtype][1])
    xd[:, :k] = to_dev(x, dtype)
    od = torch.full((m + 2, n + pads[1]), 7.0, device=DEV, dtype=TYPES[dtype][1])
    ifq.ifq_w4_gated(ifq.w4_desc(w, m, TYPES[dtype][0], R.ACTS[act], k + pads[0], n + pads[1]), xd, packed, od)
    torch.cuda.synchronize()
    assert ifq.ifq_device_status() == ifq.IFQ_OK
    assert (od[m:] == 7).all() and (od[:, n:] == 7).all()
    y, tol = R.gated(x, values[:n], values[n:], act, dtype)
    if dtype == "f16":
        tol = tol + 2.0 ** -25     # half of the smallest half
    err = np.abs(od[:m, :n].double().cpu().numpy() - y)
    assert (err <= tol).all(), np.max(err / tol)


@pytest.mark.parametrize("m", [1, 20, 300])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gated_ends_of_the_range(m, act):
    """Gate sums from -300 to 300 (x is one number a row, the weights all 1): nothing overflows on the way."""
    n, k = 24, 128
    w = ifq.w4_weights(n, k, 128, ifq.IFQ_BF16, True)
    codes, scales, mins = np.full((2 * n, k // 2), 0x11, np.uint8), np.full((2 * n, 1), 1.0), np.zeros((2 * n, 1))
    packed = pack(w, codes, scales, mins, "bf16")
    x = np.zeros((m, k))
    x[:, 5] = R.round_to(np.linspace(-300, 300, m) if m > 1 else [-200.0], "bf16")
    out = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    ifq.ifq_w4_gated(ifq.w4_desc(w, m, ifq.IFQ_BF16, R.ACTS[act]), to_dev(x, "bf16"), packed, out)
    a = x[:, 5:6]
    with np.errstate(over="ignore"):
        y = R.act(act, a) * a + np.zeros((1, n))
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    # 2^-9 for the rounding; an activation's relative error grows with |a| (the exponent's argument is rounded) to
    # |a|^2 2^-23 for a gelu's; what is below 2^-100 may be 0
    assert (np.abs(got - y) <= np.abs(y) * (2.0 ** -8 + (8 + a * a) * 2.0 ** -21) + 2.0 ** -100).all()


@pytest.mark.parametrize("m", [1, 4, 30, 200])
def test_what_is_not_finite_stays_in_its_row_and_column(m):
    n, k = 150, 264
    rng = np.random.default_rng(m)
    w = ifq.w4_weights(n, k, 32, ifq.IFQ_BF16)
    codes, scales, mins, values = draw(rng, n, k, 32, "bf16", True)
    scales[17, 3], mins[100, 8] = np.inf, np.nan       # (the last group holds 8 columns)
    packed = pack(w, codes, scales, mins, "bf16")
    x = activations(rng, m, k, "bf16", True)
    if m > 1:
        x[1, 7], x[m - 1, 263] = np.inf, np.nan
    got = matmul(w, x, packed, "bf16", "f32")
    rows, cols = np.ones(m, bool), np.ones(n, bool)
    cols[[17, 100]] = False
    if m > 1:
        rows[[1, m - 1]] = False
    assert np.array_equal(got[np.ix_(rows, cols)], (x[rows] @ values[cols].T))
    assert not np.isfinite(got[:, [17, 100]]).any() and not np.isfinite(got[~rows]).any()


@pytest.mark.parametrize("m", [1, 12, 100])
def test_residual_in_place(m):
    n, k = 200, 512
    rng = np.random.default_rng(m)
    w = ifq.w4_weights(n, k, 64, ifq.IFQ_BF16)
    codes, scales, mins, values = draw(rng, n, k, 64, "bf16", True)
    packed = pack(w, codes, scales, mins, "bf16")
    x, res = activations(rng, m, k, "bf16", True), rng.integers(-99, 99, (m, n)).astype(np.float64)
    out = to_dev(res, "bf16")
    ifq.ifq_w4_matmul(ifq.w4_desc(w, m), to_dev(x, "bf16"), packed, out, out)
    assert np.array_equal(out.double().cpu().numpy(), R.round_to(x @ values.T + res, "bf16"))


@pytest.mark.parametrize("m", [1, 3, 40, 700])
def test_same_bits_in_every_call_on_any_stream_and_in_graphs(m):
    n, k = 520, 2056
    rng = np.random.default_rng(m)
    w, g = ifq.w4_weights(n, k, 128, ifq.IFQ_BF16), ifq.w4_weights(n, k, 128, ifq.IFQ_BF16, True)
    a = draw(rng, n, k, 128, "bf16", False)
    b = draw(rng, 2 * n, k, 128, "bf16", False)
    pw, pg = pack(w, *a[:3], "bf16"), pack(g, *b[:3], "bf16")
    x = to_dev(activations(rng, m, k, "bf16", False), "bf16")

    def both():
        y, z = torch.empty(m, n, dtype=torch.bfloat16, device=DEV), torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
        ifq.ifq_w4_matmul(ifq.w4_desc(w, m), x, pw, y)
        ifq.ifq_w4_gated(ifq.w4_desc(g, m, act=1), x, pg, z)
        return y, z

    want = [t.clone() for t in both()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            got.append(both())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = both()
    for _ in range(2):
        for t in y:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got.append([t.clone() for t in y])
    assert all(torch.equal(p, q) for one in got for p, q in zip(one, want))
    assert ifq.ifq_device_status() == ifq.IFQ_OK


def test_packing_in_a_graph_before_its_product():
    n, k = 200, 392
    rng = np.random.default_rng(8)
    w = ifq.w4_weights(n, k, 64, ifq.IFQ_BF16)
    first, second = draw(rng, n, k, 64, "bf16", True), draw(rng, n, k, 64, "bf16", False)
    dev = [[torch.from_numpy(d[0]).to(DEV), to_dev(d[1], "bf16"), to_dev(d[2], "bf16")] for d in (first, second)]
    held = [t.clone() for t in dev[0]]
    x = activations(rng, 3, k, "bf16", True)
    xd, out = to_dev(x, "bf16"), torch.empty(3, n, device=DEV)
    packed = torch.empty(ifq.ifq_w4_bytes(w), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ifq.ifq_w4_pack(w, *held, packed)
        ifq.ifq_w4_matmul(ifq.w4_desc(w, 3, ifq.IFQ_F32), xd, packed, out)
    for i, d in ((0, first), (1, second), (0, first)):     # scales of 1/4 and more, then smaller ones: the flag follows
        for a, b in zip(held, dev[i]):
            a.copy_(b)
        graph.replay()
        y, tol = R.products(x, d[3])
        assert (np.abs(out.double().cpu().numpy() - y) <= tol).all()
    assert np.array_equal(out.double().cpu().numpy(), x @ first[3].T)


def test_offsets_past_32_bits():
    """Packed weights of more than 2^32 bytes, and rows of out that begin past 2^31 elements."""
    n, k = 8192 * 140, 8192
    w = ifq.w4_weights(n, k, 128, ifq.IFQ_BF16)
    size = ifq.ifq_w4_bytes(w)
    assert size > 2 ** 32
    packed = torch.zeros(size, dtype=torch.uint8, device=DEV)
    # the last rows by themselves, packed alone (their blocks are contiguous)
    rng = np.random.default_rng(0)
    tail = ifq.w4_weights(256, k, 128, ifq.IFQ_BF16)
    codes, scales, mins, values = draw(rng, 256, k, 128, "bf16", True)
    part = pack(tail, codes, scales, mins, "bf16")[:-64]
    packed[size - part.numel():] = part
    for m in (2, 40):
        x = activations(rng, m, k, "bf16", True)
        out = torch.full((m, n), 9.0, device=DEV)
        ifq.ifq_w4_matmul(ifq.w4_desc(w, m, ifq.IFQ_F32), to_dev(x, "bf16"), packed, out)
        assert np.array_equal(out[:, -256:].double().cpu().numpy(), x @ values.T)
        assert not out[:, :-256].any()
    m, small = 20, ifq.w4_weights(256, k, 128, ifq.IFQ_BF16)
    stride = 2 ** 31 // 16
    out = torch.empty(stride * m, dtype=torch.bfloat16, device=DEV)
    x = activations(rng, m, k, "bf16", True)
    ifq.ifq_w4_matmul(ifq.w4_desc(small, m, out_stride=stride), to_dev(x, "bf16"), part, out)
    got = out.view(m, stride)[:, :256].double().cpu().numpy()
    assert np.array_equal(got, R.round_to(x @ values.T, "bf16"))
