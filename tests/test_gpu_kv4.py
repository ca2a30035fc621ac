"""The paged 4-bit cache (append, read) and attention over it, against references in numpy.

Appended bytes are compared one by one: the definition rounds operation by operation.  Attention's
tolerances are derived per element beside the reference (lm_reference.attention)."""
import numpy as np
import pytest
import torch

import lm_reference as R
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"f16": (ifq.IFQ_F16, torch.float16, 2.0 ** -11), "bf16": (ifq.IFQ_BF16, torch.bfloat16, 2.0 ** -8)}
ROPES = {"none": ifq.IFQ_ROPE_NONE, "halves": ifq.IFQ_ROPE_HALVES, "pairs": ifq.IFQ_ROPE_PAIRS}


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def _status():
    torch.cuda.synchronize()
    return ifq.ifq_device_status()


# ------------------------------------------------------------------------------------ append and read


APPENDS = [
    # tokens, q heads, kv heads, D, page, dtype, rope, rot
    (1, 8, 2, 128, 16, "bf16", "halves", 128),
    (1, 1, 1, 64, 16, "f16", "none", 0),
    (7, 3, 3, 64, 48, "bf16", "pairs", 16),
    (33, 7, 1, 256, 32, "f16", "halves", 64),
    (40, 4, 2, 128, 64, "f16", "pairs", 128),
    (130, 2, 2, 256, 16, "bf16", "pairs", 256),
    (129, 5, 5, 128, 16, "bf16", "halves", 32),
    (64, 2, 1, 64, 128, "f16", "halves", 64),
    (19, 0, 2, 128, 32, "bf16", "halves", 96),
]


def _append_inputs(rng, tokens, hq, hk, D, dtype, wide):
    width = (hq + 2 * hk) * D + wide
    x = rng.normal(size=(tokens, width)).astype(np.float32)
    x[:, ::17] *= 6
    return _dev(x, TYPES[dtype][1])


@pytest.mark.parametrize("case", APPENDS)
@pytest.mark.parametrize("order", ["scattered", "in order"])
def test_append_writes_exactly_the_defined_bytes(case, order):
    tokens, hq, hk, D, page, dtype, rope, rot = case
    rng = np.random.default_rng(tokens * 7 + D)
    code, dt, _ = TYPES[dtype]
    x = _append_inputs(rng, tokens, hq, hk, D, dtype, 24)
    pages = max(3, -(-tokens // page) + 2)
    if order == "in order":
        slots = np.arange(tokens, dtype=np.int64) + page
        positions = np.arange(tokens, dtype=np.int32) + 5
    else:
        slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
        positions = rng.integers(0, tokens + 9, tokens).astype(np.int32)
        slots[tokens // 2] = -1 if tokens > 1 else slots[tokens // 2]
    rows = tokens + 9
    ang = rng.uniform(-10, 10, (rows, max(rot, 2) // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    before = rng.integers(0, 256, (pages, hk, page // 16, R.group_bytes(D))).astype(np.uint8)
    cache = _dev(before)
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hk) * D], x[:, (hq + hk) * D:(hq + 2 * hk) * D]
    pool = ifq.kv4_cache(pages, page, hk, D)
    assert ifq.ifq_kv4_cache_bytes(pool) == before.size
    q_out = torch.full((tokens, hq * D + 8), 7.0, dtype=dt, device=DEV)
    d = ifq.kv4_append_desc(pool, tokens, hq, code, ROPES[rope], rot, rows, x.shape[1], x.shape[1], x.shape[1],
                            hq * D + 8)
    ifq.ifq_kv4_append(d, q if hq else None, k, v, _dev(cos), _dev(sin), _dev(positions), _dev(slots), q_out, cache)
    assert _status() == ifq.IFQ_OK
    x32 = x.float().cpu().numpy()
    c, s = cos[positions], sin[positions]
    kr = R.rotate(x32[:, hq * D:(hq + hk) * D].reshape(tokens, hk, D), c, s, rope, rot)
    vr = x32[:, (hq + hk) * D:(hq + 2 * hk) * D].reshape(tokens, hk, D)
    want = before.copy()
    for t in range(tokens):
        for h in range(hk if slots[t] >= 0 else 0):
            R.write(want, page, slots[t], h, D, [a for a in R.quantise4(kr[t, h])], [a for a in R.quantise4(vr[t, h])])
    assert np.array_equal(cache.cpu().numpy(), want)
    if hq:
        qr = R.rotate(x32[:, :hq * D].reshape(tokens, hq, D), c, s, rope, rot).reshape(tokens, -1)
        qr = R.to_bf16(qr) if dtype == "bf16" else qr.astype(np.float16).astype(np.float32)
        assert np.array_equal(q_out[:, :hq * D].float().cpu().numpy(), qr)
    assert (q_out[:, hq * D:] == 7).all()
    # and read back
    ko, vo = (torch.full((tokens, hk * D), 3.0, dtype=dt, device=DEV) for _ in range(2))
    ifq.ifq_kv4_read(d, cache, _dev(slots), ko, vo)
    assert _status() == ifq.IFQ_OK
    (kv, _, _), (vv, _, _) = R.read(want, page, np.maximum(slots, 0), D)
    for got, val in ((ko, kv), (vo, vv)):
        val = np.where(slots[:, None, None] >= 0, val, 0).astype(np.float32).reshape(tokens, -1)
        val = R.to_bf16(val) if dtype == "bf16" else val.astype(np.float16).astype(np.float32)
        assert np.array_equal(got.float().cpu().numpy(), val)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_append_of_rows_that_are_constant_huge_or_not_finite(D):
    hk, page = 1, 16
    rows = np.zeros((7, D), np.float32)
    rows[0] = 2.5                                   # constant: scale 0
    rows[1] = np.linspace(-3e38, 3e38, D)           # clamped
    rows[2, 3] = np.inf
    rows[3, D - 1] = -np.inf
    rows[4, 5] = np.nan
    rows[5] = np.linspace(0, 1e-7, D)               # steps below half's range
    rows[6, 7] = -65504.0 * 2
    x = _dev(rows, torch.bfloat16)
    cache = torch.zeros(1, hk, 1, R.group_bytes(D), dtype=torch.uint8, device=DEV)
    d = ifq.kv4_append_desc(ifq.kv4_cache(1, page, hk, D), 7, 0, ifq.IFQ_BF16, ifq.IFQ_ROPE_NONE)
    ifq.ifq_kv4_append(d, None, x, x, None, None, None, torch.arange(7, device=DEV), None, cache)
    assert _status() == ifq.IFQ_OK
    x32, got = x.float().cpu().numpy(), cache.cpu().numpy()
    want = np.zeros_like(got)
    for t in (0, 1, 2, 3, 5, 6):
        kq = R.quantise4(x32[t])
        R.write(want, page, t, 0, D, kq, kq)
    (kv, _, kp), _ = R.read(got, page, np.arange(7), D)
    assert np.isnan(kp[4].astype(np.float32)).all() and np.isnan(kv[4]).all()
    sel = [0, 1, 2, 3, 5, 6]
    (kw, _, _), (vw, _, _) = R.read(want, page, np.arange(7), D)
    (_, _, _), (vv, _, _) = R.read(got, page, np.arange(7), D)
    assert np.array_equal(kv[sel], kw[sel]) and np.array_equal(vv[sel], vw[sel])


def test_append_in_place_and_on_another_stream():
    rng = np.random.default_rng(3)
    hq, hk, D, page, tokens = 4, 2, 128, 32, 21
    x = _append_inputs(rng, tokens, hq, hk, D, "f16", 0)
    ang = rng.uniform(-3, 3, (tokens, D // 2))
    cos, sin, pos = _dev(np.cos(ang).astype(np.float32)), _dev(np.sin(ang).astype(np.float32)), torch.arange(
        tokens, dtype=torch.int32, device=DEV)
    slots = torch.arange(tokens, device=DEV)
    pool = ifq.kv4_cache(1, page, hk, D)
    W = x.shape[1]
    outs = []
    for inplace in (False, True):
        y = x.clone()
        cache = torch.zeros(1, hk, 2, R.group_bytes(D), dtype=torch.uint8, device=DEV)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        q_out = y if inplace else torch.empty(tokens, hq * D, dtype=torch.float16, device=DEV)
        d = ifq.kv4_append_desc(pool, tokens, hq, ifq.IFQ_F16, ifq.IFQ_ROPE_HALVES, D, tokens, W, W, W,
                                W if inplace else 0)
        ifq.ifq_kv4_append(d, y, y[:, hq * D:], y[:, (hq + hk) * D:], cos, sin, pos, slots, q_out, cache, stream=st)
        st.synchronize()
        outs.append((q_out[:, :hq * D].clone(), cache))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_bad_slots_and_positions_are_reported_and_skipped():
    hk, D, page = 1, 64, 16
    cache = torch.zeros(2, hk, 1, R.group_bytes(D), dtype=torch.uint8, device=DEV)
    x = torch.randn(3, D, device=DEV).half()
    tab = torch.ones(4, D // 2, device=DEV)
    pool = ifq.kv4_cache(2, page, hk, D)
    d = ifq.kv4_append_desc(pool, 3, 0, ifq.IFQ_F16, ifq.IFQ_ROPE_HALVES, D, 4)
    for slots, pos in (([1, 32, 2], [0, 1, 2]), ([1, 1 << 40, 2], [0, 1, 2]), ([1, 3, 2], [0, 4, 2]), ([1, 3, 2], [0, -1, 2])):
        cache.zero_()
        ifq.ifq_kv4_append(d, None, x, x, tab, tab, torch.tensor(pos, dtype=torch.int32, device=DEV),
                           torch.tensor(slots, device=DEV), None, cache)
        assert _status() == ifq.IFQ_ERANGE
        params = cache.view(2, -1)[0, 16 * D:].view(torch.int32)[:16].cpu()
        assert params[1] != 0 and params[2] != 0 and (params[[0, 3]] == 0).all()
        assert not cache[1].any()
    out = torch.full((3, D), 9.0, dtype=torch.float16, device=DEV)
    ifq.ifq_kv4_read(d, cache, torch.tensor([1, 32, -5], device=DEV), out)
    assert _status() == ifq.IFQ_ERANGE
    assert out[0].any() and not out[1:].any()
    assert _status() == ifq.IFQ_OK


# ------------------------------------------------------------------------------------ attention


def _setup(rng, lens, nq, hq, hk, D, page, garbage=0xFF, spread=1.0, spare=2, first_page=0):
    """A cache whose bytes are `garbage` (0xFF: NaN parameters) but for the sequences' tokens, on pages in any order,
    and a table whose unused entries are out of range."""
    lens = np.asarray(lens, np.int32)
    starts = np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)
    need = -(-lens // page)
    pages = int(need.sum()) + spare
    row = max(1, int(need.max()) + 1)
    table = np.full((len(lens), row), -7, np.int32)
    perm = rng.permutation(pages)
    at = 0
    cache = np.full((pages, hk, page // 16, R.group_bytes(D)), garbage, np.uint8)
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n]
        at += n
        j = np.arange(lens[s])
        R.fill(rng, cache, page, table[s, j // page].astype(np.int64) * page + j % page, D, spread)
    table[table >= 0] += first_page
    q = rng.normal(size=(int(starts[-1]), hq, D)).astype(np.float32) * 1.5
    return lens, starts, table, cache, q


def _run(lens, starts, table, cache, q, hq, hk, D, page, dtype, window=0, sinks=0, scale=None, max_q=None, max_len=0,
         pad=0, use_starts=True, lse=True, cache_dev=None, pages=None, stream=None, wide=False):
    """wide: bounds as for long sequences with many queries, which choose other kernels and launch shapes."""
    code, dt, u = TYPES[dtype]
    scale = D ** -0.5 if scale is None else scale
    T = q.shape[0]
    if wide:
        table = np.concatenate([table, np.full((len(table), 200000 // page), -3, np.int32)], 1)
        max_q = max(300, int(np.diff(starts).max())) if max_q is None else max_q
    qd = torch.zeros(T, hq * D + pad, dtype=dt, device=DEV)
    qd[:, :hq * D] = _dev(q.reshape(T, -1), dt)
    out = torch.full((T, hq * D + pad), 5.0, dtype=dt, device=DEV)
    ls = torch.full((T, hq), 5.0, device=DEV)
    pool = ifq.kv4_cache(pages or cache.shape[0], page, hk, D)
    d = ifq.kv4_attention_desc(pool, len(lens), T, int(np.diff(starts).max()) if max_q is None else max_q,
                               table.shape[1], hq, code, scale, window, sinks, max_len, hq * D + pad, hq * D + pad)
    size = ifq.ifq_kv4_attention_workspace_bytes(d)
    ws = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    args = (d, qd, _dev(cache) if cache_dev is None else cache_dev, _dev(table), _dev(lens),
            _dev(starts) if use_starts else None, out, ls if lse else None, ws, size)
    torch.cuda.synchronize()
    ifq.ifq_kv4_attention(*args, stream=stream)
    torch.cuda.synchronize()
    first = out.clone(), ls.clone()
    for _ in range(2):     # the same again, whatever the workspace holds now
        ifq.ifq_kv4_attention(*args, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(first[0].view(torch.int16), out.view(torch.int16))
    if lse:
        assert torch.equal(first[1].view(torch.int32), ls.view(torch.int32))
    assert (out[:, hq * D:] == 5).all()
    q64 = qd[:, :hq * D].double().cpu().numpy().reshape(T, hq, D)
    many = dtype == "bf16" and d.max_q * (hq // hk) > 32     # the library then rounds values to half
    return (out[:, :hq * D].double().cpu().numpy().reshape(T, hq, D), ls.double().cpu().numpy(), q64, scale, u, many)


def _check(got, lens, starts, table, cache, hk, page, window=0, sinks=0, rows=None, lse=True):
    out, ls, q64, scale, u, many = got
    want, wl, tol, ltol = R.attention(q64, cache, page, table, lens, starts, hk, scale, window, sinks, u, many)
    rows = slice(None) if rows is None else rows
    with np.errstate(all="ignore"):
        far = np.abs(out[rows] - want[rows]) - tol[rows]
        assert not np.isnan(far).any() and (far <= 0).all(), (np.nanmax(far), np.argwhere(~(far <= 0))[:5])
        if lse:
            empty = np.isneginf(wl[rows])
            assert np.array_equal(np.isneginf(ls[rows]), empty)
            far = np.where(empty, 0, np.abs(np.where(empty, 0, ls[rows]) - np.where(empty, 0, wl[rows])) - ltol[rows])
            assert (far <= 0).all(), np.nanmax(far)


CASES = [
    # lens, queries, q heads, kv heads, D, page, dtype, window, sinks
    ([1], [1], 1, 1, 64, 16, "f16", 0, 0),
    ([0, 1, 2, 15, 16, 17], [1] * 6, 8, 2, 128, 16, "bf16", 0, 0),
    ([31, 32, 33, 250, 0, 64], [1] * 6, 4, 4, 64, 32, "f16", 0, 0),
    ([100, 37, 700], [1] * 3, 7, 1, 256, 48, "bf16", 0, 0),
    ([500, 3], [1, 1], 16, 1, 128, 64, "f16", 0, 0),
    ([1100], [1], 32, 2, 128, 16, "bf16", 0, 0),
    ([129, 40, 5, 80], [5, 0, 5, 3], 8, 1, 128, 16, "f16", 0, 0),
    ([60, 16, 300], [4, 16, 7], 6, 2, 64, 16, "bf16", 0, 0),
    ([200, 90], [2, 9], 24, 2, 256, 32, "f16", 0, 0),
    ([600, 20, 99], [1] * 3, 8, 2, 128, 16, "bf16", 64, 4),
    ([600, 20, 99], [1] * 3, 8, 2, 64, 16, "f16", 1, 0),
    ([600, 333], [6, 2], 4, 2, 128, 16, "f16", 50, 20),
    ([700], [9], 4, 1, 128, 16, "bf16", 33, 1),
    ([40, 300], [3, 33], 4, 2, 64, 16, "bf16", 500, 500),
    ([150, 1, 70], [70, 1, 70], 4, 2, 128, 16, "bf16", 0, 0),
    ([333, 200], [200, 131], 8, 2, 64, 64, "f16", 0, 0),
    ([140, 129], [129, 129], 5, 1, 128, 32, "f16", 40, 3),
    ([260], [66], 2, 1, 256, 16, "bf16", 0, 0),
    ([400, 0, 385], [130, 1, 128], 8, 4, 128, 128, "bf16", 0, 0),
    ([3, 2], [5, 2], 4, 2, 128, 16, "f16", 0, 0),      # more queries than tokens: the first see nothing
    ([40], [64], 2, 1, 64, 16, "bf16", 7, 2),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_attention_equals_its_definition(case, wide):
    lens, nq, hq, hk, D, page, dtype, window, sinks = case
    rng = np.random.default_rng(sum(lens) + hq)
    lens, starts, table, cache, q = _setup(rng, lens, nq, hq, hk, D, page)
    got = _run(lens, starts, table, cache, q, hq, hk, D, page, dtype, window, sinks, pad=8 if hq % 2 else 0, wide=wide)
    assert _status() == ifq.IFQ_OK
    _check(got, lens, starts, table, cache, hk, page, window, sinks)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("D,hq,hk,n", [(128, 8, 2, 1), (64, 4, 1, 3), (128, 4, 1, 80), (256, 2, 1, 40)])
def test_attention_of_peaked_and_of_flat_scores(D, hq, hk, n, wide):
    """Scores that differ by hundreds (one token takes everything), and scores that are all the same."""
    rng = np.random.default_rng(5)
    lens, starts, table, cache, q = _setup(rng, [450], [n], hq, hk, D, 16, spread=3.0)
    for scale in (8.0, 0.0, -0.3):
        got = _run(lens, starts, table, cache, q, hq, hk, D, 16, "bf16", scale=scale, wide=wide)
        _check(got, lens, starts, table, cache, hk, 16)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n,dtype", [(1, "f16"), (90, "f16"), (90, "bf16")])
def test_attention_of_values_of_very_different_sizes(n, dtype, wide):
    """Value scales over 20 binary orders, ascending and descending along the sequence: nothing that matters is lost
    in the weights' half precision."""
    rng = np.random.default_rng(6)
    D, page, hk, hq, L = 128, 16, 1, 4, 320
    for down in (False, True):
        lens, starts, table, cache, q = _setup(rng, [L], [n], hq, hk, D, page)
        for j in range(L):
            pg, off = table[0, j // page], j % page
            sc = np.float16(2.0 ** (-14 + 20 * ((L - 1 - j) if down else j) / (L - 1)))
            g = cache[pg, 0, off // 16]
            g[16 * D + 64 + 4 * (off % 16):16 * D + 68 + 4 * (off % 16)] = np.array([sc, -3 * sc], np.float16).view(np.uint8)
        got = _run(lens, starts, table, cache, q, hq, hk, D, page, dtype, wide=wide)
        _check(got, lens, starts, table, cache, hk, page)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n", [1, 70])
def test_attention_of_tiny_and_huge_queries(n, wide):
    rng = np.random.default_rng(7)
    D, page, hk, hq = 128, 16, 2, 4
    lens, starts, table, cache, q = _setup(rng, [200], [n], hq, hk, D, page)
    q[:, 0] *= 1e-30
    q[:, 1] *= 3e4
    q[:, 2] = 0
    q[:, 3, ::2] *= 1e-6
    got = _run(lens, starts, table, cache, q, hq, hk, D, page, "bf16", wide=wide)
    _check(got, lens, starts, table, cache, hk, page)


@pytest.mark.parametrize("dtype,wide", [("bf16", False), ("bf16", True), ("f16", True)])
@pytest.mark.parametrize("n", [1, 4, 100])
def test_what_is_not_finite_stays_where_it_is_seen(n, dtype, wide):
    """A NaN query row makes its own output NaN alone; a NaN token those of the rows that see it."""
    rng = np.random.default_rng(8)
    D, page, hk, hq = 128, 16, 2, 4
    lens, starts, table, cache, q = _setup(rng, [210, 180], [n, n], hq, hk, D, page)
    q2 = q.copy()
    q2[0, 1, 3] = np.nan
    got = _run(lens, starts, table, cache, q2, hq, hk, D, page, dtype, wide=wide)
    assert np.isnan(got[0][0, 1]).all()
    keep = np.ones(got[0].shape[:2], bool)
    keep[0, 1] = False
    _check(got, lens, starts, table, cache, hk, page, rows=keep)
    # token 209 of the first sequence is seen by its last query alone
    c2 = cache.copy()
    pg, off = table[0, 209 // page], 209 % page
    c2[pg, 0, off // 16][16 * D + 4 * (off % 16):16 * D + 4 * (off % 16) + 4] = 0xFF
    c2[pg, 0, off // 16][16 * D + 64 + 4 * (off % 16):16 * D + 68 + 4 * (off % 16)] = 0xFF
    got = _run(lens, starts, table, c2, q, hq, hk, D, page, dtype, wide=wide)
    assert np.isnan(got[0][n - 1, :2]).all()
    keep = np.ones(got[0].shape[:2], bool)
    keep[n - 1, :2] = False
    _check(got, lens, starts, table, cache, hk, page, rows=keep)


@pytest.mark.parametrize("bounds", [dict(max_q=300), dict(max_len=2000), dict(max_q=1024, max_len=650)])
def test_generous_bounds_change_nothing_that_matters(bounds):
    rng = np.random.default_rng(9)
    lens, starts, table, cache, q = _setup(rng, [640, 33], [3, 2], 8, 2, 128, 64)
    table = np.concatenate([table, np.full((2, 40), 1 << 30, np.int32)], 1)
    got = _run(lens, starts, table, cache, q, 8, 2, 128, 64, "f16", **bounds)
    _check(got, lens, starts, table, cache, 2, 64)


def test_one_query_a_sequence_without_starts_and_without_lse():
    rng = np.random.default_rng(10)
    lens, starts, table, cache, q = _setup(rng, [5, 70, 33], [1] * 3, 8, 4, 64, 16)
    got = _run(lens, starts, table, cache, q, 8, 4, 64, 16, "bf16", use_starts=False, lse=False)
    _check(got, lens, starts, table, cache, 4, 16, lse=False)


@pytest.mark.parametrize("n,wide", [(1, False), (5, False), (65, False), (5, True), (65, True)])
def test_many_sequences(n, wide):
    """More sequences than a block has threads, lengths from none to a few pages."""
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 40, 1030)
    nq = np.minimum(rng.integers(0, 2, 1030), 1) * n
    nq[:2] = n
    lens, starts, table, cache, q = _setup(rng, lens, nq, 2, 1, 64, 16)
    got = _run(lens, starts, table, cache, q, 2, 1, 64, 16, "f16", wide=wide)
    assert _status() == ifq.IFQ_OK
    _check(got, lens, starts, table, cache, 1, 16)


@pytest.mark.parametrize("n,wide", [(1, False), (3, False), (72, False), (1, True), (72, True)])
def test_pages_past_four_gigabytes(n, wide):
    rng = np.random.default_rng(12)
    D, page, hk, hq = 128, 64, 2, 4
    lens, starts, table, cache, q = _setup(rng, [300], [n], hq, hk, D, page, spare=0)
    per = hk * (page // 16) * R.group_bytes(D)
    first = (1 << 32) // per + 3
    big = torch.empty((first + cache.shape[0], hk, page // 16, R.group_bytes(D)), dtype=torch.uint8, device=DEV)
    big[first:] = _dev(cache)
    got = _run(lens, starts, np.where(table >= 0, table + first, table).astype(np.int32), cache, q, hq, hk, D, page, "bf16",
               cache_dev=big, pages=big.shape[0], wide=wide)
    _check(got, lens, starts, table, cache, hk, page)


@pytest.mark.parametrize("n,wide", [(1, False), (80, False), (1, True), (80, True)])
def test_bad_lengths_starts_and_pages_are_reported(n, wide):
    rng = np.random.default_rng(13)
    D, page, hk, hq = 64, 16, 1, 2
    lens, starts, table, cache, q = _setup(rng, [120, 130, 90], [n] * 3, hq, hk, D, page)
    others = np.ones((3 * n, hq), bool)
    others[n:2 * n] = False
    for what in ("long", "negative", "page", "low page"):
        l2, t2 = lens.copy(), table.copy()
        if what == "long":
            l2[1] = (table.shape[1] + 200000) * page + 1
        elif what == "negative":
            l2[1] = -1
        else:
            t2[1, 2] = cache.shape[0] if what == "page" else -1
        got = _run(l2, starts, t2, cache, q, hq, hk, D, page, "f16", wide=wide)
        assert _status() == ifq.IFQ_ERANGE, what
        _check(got, lens, starts, table, cache, hk, page, rows=others)
        if what in ("long", "negative"):
            assert (got[0][n:2 * n] == 5).all()
    for st in ([0, n, n - 1, 3 * n], [0, n, 2 * n, 3 * n + 1]):
        _run(lens, np.array(st, np.int32), table, cache, q, hq, hk, D, page, "f16", max_q=n, wide=wide)
        assert _status() == ifq.IFQ_ERANGE
    _run(lens, starts, table, cache, q, hq, hk, D, page, "f16", max_q=n - 1, wide=wide)
    assert _status() == ifq.IFQ_ERANGE


def test_attention_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(14)
    lens, starts, table, cache, q = _setup(rng, [900, 40], [1, 1], 8, 2, 128, 32)
    want = _run(lens, starts, table, cache, q, 8, 2, 128, 32, "bf16")[0]
    st = torch.cuda.Stream()
    got = _run(lens, starts, table, cache, q, 8, 2, 128, 32, "bf16", stream=st)[0]
    assert np.array_equal(want, got)
    # captured once, replayed on new inputs
    dt = torch.bfloat16
    qd, cd, td, ld = _dev(q.reshape(2, -1), dt), _dev(cache), _dev(table), _dev(lens)
    out = torch.zeros_like(qd)
    d = ifq.kv4_attention_desc(ifq.kv4_cache(cache.shape[0], 32, 2, 128), 2, 2, 1, table.shape[1], 8, ifq.IFQ_BF16,
                               128 ** -0.5)
    size = ifq.ifq_kv4_attention_workspace_bytes(d)
    ws = torch.zeros(max(size, 16), dtype=torch.uint8, device=DEV)
    ifq.ifq_kv4_attention(d, qd, cd, td, ld, None, out, None, ws, size)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ifq.ifq_kv4_attention(d, qd, cd, td, ld, None, out, None, ws, size)
    for l in ([900, 40], [17, 33], [899, 1]):
        ld.copy_(torch.tensor(l, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want = _run(np.array(l, np.int32), starts, table, cache, q, 8, 2, 128, 32, "bf16")[0]
        assert np.array_equal(out.double().cpu().numpy().reshape(2, 8, 128), want)


def test_nothing_to_do():
    rng = np.random.default_rng(15)
    lens, starts, table, cache, q = _setup(rng, [20], [1], 2, 1, 64, 16)
    pool = ifq.kv4_cache(cache.shape[0], 16, 1, 64)
    x = torch.full((1, 128), 5.0, device=DEV).half()
    for seqs, T in ((0, 0), (1, 0)):
        d = ifq.kv4_attention_desc(pool, seqs, T, 1, table.shape[1], 2, ifq.IFQ_F16, 1.0)
        ws = torch.zeros(max(16, ifq.ifq_kv4_attention_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
        ifq.ifq_kv4_attention(d, x, _dev(cache), _dev(table), _dev(lens), torch.zeros(2, dtype=torch.int32, device=DEV), x,
                              None, ws, ws.numel())
    assert _status() == ifq.IFQ_OK and (x == 5).all()
    d = ifq.kv4_append_desc(pool, 0, 2, ifq.IFQ_F16, ifq.IFQ_ROPE_NONE)
    ifq.ifq_kv4_append(d, x, x, x, None, None, None, x, x, _dev(cache))
    ifq.ifq_kv4_read(d, _dev(cache), x, x, x)
    assert _status() == ifq.IFQ_OK and (x == 5).all()
