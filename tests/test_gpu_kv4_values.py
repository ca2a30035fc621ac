"""Attention over values of mixed sizes, constant value rows, dominant tokens and parameters that are no numbers.

Tolerances are those of lm_reference.attention, whose term for rounded weights goes with s' c' + |m'|; the kernels round the
weights of c' - 8 (|c' - 8| <= 8) and add the minima unrounded, which the term of _near adds: 2^-11 of sum p 8 s' / sum p."""
import numpy as np
import pytest
import torch

import lm_reference as R
import test_gpu_kv4 as base
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu


def _value(cache, table, page, D, seq, j, scale, mn, code=None):
    """Value parameters of token j (all heads), and one code for all dimensions if given."""
    pg, off = table[seq, j // page], j % page
    g, row = cache[pg, :, off // 16], off % 16
    g[:, 16 * D + 64 + 4 * row:16 * D + 68 + 4 * row] = np.array([scale, mn], np.float16).view(np.uint8)
    if code is not None:
        byte, shift = R.v_place(D)
        low, high = byte[row][shift[row] == 0], byte[row][shift[row] == 4]
        assert np.array_equal(low, high)
        g[:, low] = code | code << 4


def _key(cache, table, page, D, seq, j, value):
    """A key with every element `value` (scale 0)."""
    pg, off = table[seq, j // page], j % page
    g, row = cache[pg, :, off // 16], off % 16
    g[:, 16 * D + 4 * row:16 * D + 4 * row + 4] = np.array([0, value], np.float16).view(np.uint8)


def _near(got, lens, starts, table, cache, hk, page, rows=None, lse=True, window=0, sinks=0):
    out, ls, q64, scale, u, many = got
    want, wl, tol, ltol = R.attention(q64, cache, page, table, lens, starts, hk, scale, window, sinks, u, many)
    # the same attention over 8 s' in place of the values: its mean, and the largest
    eight = cache.copy()
    D = q64.shape[2]
    par = eight[..., 16 * D + 64:].reshape(-1, 16, 4).view(np.float16)
    with np.errstate(all="ignore"):
        par[..., 1] = np.where(np.isfinite(par[..., 0]), 8 * par[..., 0], 0)
    par[..., 0] = 0
    eight[..., 16 * D + 64:] = par.view(np.uint8).reshape(*eight.shape[:-1], 64)
    mean, _, _, _ = R.attention(q64, eight, page, table, lens, starts, hk, scale, window, sinks, 0.0)
    with np.errstate(all="ignore"):
        tol = tol + 2.0 ** -11 * mean
    keep = np.ones(out.shape[:2], bool) if rows is None else rows
    far = np.abs(out[keep] - want[keep]) - tol[keep]
    assert (far <= 0).all(), (np.nanmax(far), np.isnan(far).sum(), np.argwhere(~(far <= 0))[:5])
    if lse:
        far = np.abs(ls[keep] - wl[keep]) - ltol[keep]
        assert (far <= 0).all(), (np.nanmax(far), np.isnan(far).sum())


MANY = [dict(), dict(wide=True), dict(wide=True, max_q=30)]     # by estimate; wide row blocks; 128 rows a block, split keys


@pytest.mark.parametrize("bounds", MANY, ids=["as is", "wide", "wide 30"])
@pytest.mark.parametrize("n,dtype", [(1, "f16"), (30, "f16"), (30, "bf16")])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", ["constant rows", "scales to 1", "scales to 64"])
def test_values_with_minima_that_do_not_go_with_their_scales(kind, D, n, dtype, bounds):
    """Every other value row constant (scale 0, codes 0, as the append writes them) beside usual ones, or scales from 0 and
    2^-24 up: what a token adds does not depend on how small its scale is."""
    rng = np.random.default_rng(21)
    page, hk, hq, L = 16, 1, 4, 300
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    top = {"constant rows": 0, "scales to 1": 0, "scales to 64": 6}[kind]
    for j in range(L):
        if j % 2:
            _value(cache, table, page, D, 0, j, 0, rng.uniform(1, 5), 0)
        elif kind == "constant rows":
            _value(cache, table, page, D, 0, j, 0.5, -3.75)
        else:
            _value(cache, table, page, D, 0, j, 2.0 ** rng.uniform(-24, top), 5.0)
    got = base._run(lens, starts, table, cache, q, hq, hk, D, page, dtype, **bounds)
    _near(got, lens, starts, table, cache, hk, page)


@pytest.mark.parametrize("bounds", MANY[1:], ids=["wide", "wide 30"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("last", [24.6, 26.5, 29.5])
def test_a_maximum_that_rises_by_many_binades_within_a_tile(last, D, dtype, bounds):
    """Tokens 0 to 31 of the first tile at score 2^0, the next 64 at 2^11.5 (2^14 for f16), token 96 at 2^last, whose value
    is 0: what the 64 add is all there is to see."""
    rng = np.random.default_rng(22)
    page, hk, hq, L, n = 16, 1, 4, 200, 30
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    q[:] = 0
    q[:, :, 0] = 1
    for j in range(L):
        _key(cache, table, page, D, 0, j, 0.0 if not 32 <= j <= 96 else last if j == 96 else 14.0 if dtype == "f16" else 11.5)
        _value(cache, table, page, D, 0, j, 0.25, 1.0)
    if dtype == "f16":
        _value(cache, table, page, D, 0, 96, 0.25, -2.0, 8)
    else:
        _value(cache, table, page, D, 0, 96, 0.0, 0.0, 0)
    got = base._run(lens, starts, table, cache, q, hq, hk, D, page, dtype, scale=float(np.float32(np.log(2))), **bounds)
    _near(got, lens, starts, table, cache, hk, page)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n,dtype", [(1, "bf16"), (5, "f16"), (60, "bf16"), (60, "f16")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_page_past_the_cache_does_not_bring_in_what_another_call_left(D, n, dtype, wide):
    """The values of such a page are undefined, but the same each time: nothing of the calls before shows in them."""
    rng = np.random.default_rng(27)
    page, hk, hq, L = 16, 1, 2, 700
    a = base._setup(rng, [L], [n], hq, hk, D, page)
    bad = a[2].copy()
    bad[0, 2::5] = a[3].shape[0] + 3
    outs = []
    for spread in (0.5, 2.0, 7.0):
        other = base._setup(rng, [L, L], [n, n], hq, hk, D, page, spread=spread)
        base._run(*other, hq, hk, D, page, dtype, wide=wide)
        got = base._run(a[0], a[1], bad, a[3], a[4], hq, hk, D, page, dtype, wide=wide)
        assert base._status() == ifq.IFQ_ERANGE
        outs.append(got)
    for o in outs[1:]:
        assert np.array_equal(o[0], outs[0][0], equal_nan=True) and np.array_equal(o[1], outs[0][1], equal_nan=True)


@pytest.mark.parametrize("bounds", MANY, ids=["as is", "wide", "wide 30"])
@pytest.mark.parametrize("n,dtype", [(1, "bf16"), (4, "f16"), (4, "bf16"), (30, "f16"), (30, "bf16")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_value_that_is_not_a_number_leaves_the_log_sum_exp(D, n, dtype, bounds):
    rng = np.random.default_rng(24)
    page, hk, hq, L = 16, 1, 4, 150
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    c2 = cache.copy()
    _value(c2, table, page, D, 0, L - 2, np.nan, np.nan)        # seen by the last two queries
    got = base._run(lens, starts, table, c2, q, hq, hk, D, page, dtype, **bounds)
    sees = np.arange(n) >= n - 2
    assert np.isnan(got[0][sees]).all()
    rows = np.broadcast_to(~sees[:, None], got[0].shape[:2])
    _near(got, lens, starts, table, cache, hk, page, rows=rows)
    _, wl, _, ltol = R.attention(got[2], cache, page, table, lens, starts, hk, got[3], 0, 0, got[4], got[5])
    assert (np.abs(got[1] - wl) <= ltol).all()


@pytest.mark.parametrize("bounds", MANY[1:], ids=["wide", "wide 30"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("binades", [20.0, 24.5, 26.0, 28.0])
def test_a_first_token_that_dominates_and_holds_nothing(binades, D, dtype, bounds):
    """A first token with almost all of the weight and a value of 0.  The others' weights lie `binades` below: a reference
    ten binades below the first maximum leaves them 2^-25 / 2^9 of it as the step of half's subnormals."""
    rng = np.random.default_rng(23)
    page, hk, hq, L, n = 16, 1, 4, 260, 30
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    q[:] = 0
    q[:, :, 0] = 1
    for j in range(L):
        _key(cache, table, page, D, 0, j, binades if j == 0 else 0.0)
    if dtype == "f16":
        _value(cache, table, page, D, 0, 0, 0.25, -2.0, 8)
    else:
        _value(cache, table, page, D, 0, 0, 0.0, 0.0, 0)
    got = base._run(lens, starts, table, cache, q, hq, hk, D, page, dtype, scale=float(np.float32(np.log(2))), **bounds)
    out, ls, q64, scale, u, many = got
    # by hand: the terms of lm_reference.attention for all but the first token, whose weight is exact and whose value is 0
    (_, (v, vc, vp)) = R.read(cache, page, table[0, np.arange(L) // page].astype(np.int64) * page + np.arange(L) % page, D)
    v, s8 = v[:, 0], 8 * vp[:, 0, 0].astype(np.float64)
    mag = np.abs(v).max(1) + s8
    p = np.exp(np.where(np.arange(L) == 0, binades, 0.0) * scale - binades * scale)
    delta = (D + 8) * 2.0 ** -23 * binades * scale
    for i in range(n):
        m = L - n + 1 + i
        w = p[:m] / p[:m].sum()
        want = w @ v[:m]
        others = (w[1:] * mag[1:m]).sum()
        tol = u * np.abs(want) + (2 * delta + 2.0 ** -10 + 2 * m * 2.0 ** -24) * others + m * 2.0 ** -34 * mag[:m].max() + 2.0 ** -24 * w[1:].sum()
        tol = tol + (2.0 ** -25 if dtype == "f16" else 0)       # results below half's normal range
        far = np.abs(out[i] - want) - tol
        assert (far <= 0).all(), (i, far.max(), tol.max(), np.abs(want).max())


@pytest.mark.parametrize("bounds", MANY, ids=["as is", "wide", "wide 30"])
@pytest.mark.parametrize("n,dtype", [(2, "f16"), (4, "bf16"), (30, "f16"), (30, "bf16")])
@pytest.mark.parametrize("what", ["scale", "min", "both"])
def test_an_infinite_value_reaches_only_the_rows_that_see_it(what, n, dtype, bounds):
    rng = np.random.default_rng(25)
    page, hk, hq, L, D = 16, 2, 4, 210, 128
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    c2 = cache.copy()
    _value(c2, table, page, D, 0, L - 1, np.inf if what != "min" else 0.2, np.inf if what != "scale" else -1.5)
    got = base._run(lens, starts, table, c2, q, hq, hk, D, page, dtype, **bounds)
    assert not np.isfinite(got[0][n - 1]).any()
    rows = np.ones(got[0].shape[:2], bool)
    rows[n - 1] = False
    _near(got, lens, starts, table, cache, hk, page, rows=rows)


@pytest.mark.parametrize("bounds", MANY, ids=["as is", "wide", "wide 30"])
@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_values_below_the_normal_range_of_half(D, n, bounds):
    """Scales of a few dozen times 2^-24, in bfloat16: rounding a value to half takes 2^-24 of it at most, and half of its
    minimum as much again."""
    rng = np.random.default_rng(26)
    page, hk, hq, L = 16, 1, 4, 200
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    for j in range(L):
        k = 4 * int(rng.integers(1, 15)) + 1
        _value(cache, table, page, D, 0, j, k * 2.0 ** -24, -7 * k * 2.0 ** -24)
    got = base._run(lens, starts, table, cache, q, hq, hk, D, page, "bf16", **bounds)
    out, ls, q64, scale, u, many = got
    want, wl, tol, ltol = R.attention(q64, cache, page, table, lens, starts, hk, scale, 0, 0, u, many)
    far = np.abs(out - want) - tol - 2.0 ** -24
    assert (far <= 0).all(), (far.max(), tol.max())


@pytest.mark.parametrize("bounds", MANY, ids=["as is", "wide", "wide 30"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("at,seen", [(60, 0), (100, 20), (1, 30), (3, 0)])
def test_a_value_that_is_not_a_number_beside_a_window(at, seen, dtype, bounds):
    """Queries at 120 to 149 see their last 40 tokens and the first three: token 60 is seen by none, 100 by those below 140."""
    rng = np.random.default_rng(28)
    page, hk, hq, L, n, D = 32, 2, 8, 150, 30, 128
    lens, starts, table, cache, q = base._setup(rng, [L], [n], hq, hk, D, page)
    c2 = cache.copy()
    _value(c2, table, page, D, 0, at, np.nan, 0.5)
    got = base._run(lens, starts, table, c2, q, hq, hk, D, page, dtype, 40, 3, **bounds)
    assert np.isnan(got[0][:seen]).all()
    rows = np.broadcast_to((np.arange(n) >= seen)[:, None], got[0].shape[:2])
    _near(got, lens, starts, table, cache, hk, page, rows=rows, window=40, sinks=3)
    _, wl, _, ltol = R.attention(got[2], cache, page, table, lens, starts, hk, got[3], 40, 3, got[4], got[5])
    assert (np.abs(got[1] - wl) <= ltol).all()
