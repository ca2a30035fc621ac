"""Refusals and sizes of the decoder layer's operators: argument errors come back before anything is launched (no GPU)."""
import pytest

from paper_1911_08076_gb300 import ifq

FAKE = 1 << 20     # never dereferenced
E = ifq
BIG = 2 ** 31 - 1


def _status(f, *a, **k):
    with pytest.raises(ifq.IfqError) as e:
        f(*a, **k)
    return e.value.status


def test_packed_sizes():
    """16 x 128 blocks of 1024 bytes and 64 a group, rows up to whole tiles of 128; 64 bytes behind them."""
    assert ifq.ifq_w4_bytes(ifq.w4_weights(4096, 4096, 128)) == 256 * 32 * 1088 + 64
    assert ifq.ifq_w4_bytes(ifq.w4_weights(1, 8, 32)) == 8 * 1280 + 64
    assert ifq.ifq_w4_bytes(ifq.w4_weights(65, 136, 64, gated=True)) == 16 * 2 * 1152 + 64
    assert ifq.ifq_w4_bytes(ifq.w4_weights(131072, 65536, 128)) == 8192 * 512 * 1088 + 64


@pytest.mark.parametrize("change,status", [
    (dict(n=0), E.IFQ_EINVAL), (dict(k=0), E.IFQ_EINVAL), (dict(n=-5), E.IFQ_EINVAL), (dict(k=12), E.IFQ_ESHAPE),
    (dict(group=16), E.IFQ_EUNSUPPORTED), (dict(group=0), E.IFQ_EUNSUPPORTED), (dict(dtype=ifq.IFQ_F32), E.IFQ_EINVAL),
    (dict(dtype=0), E.IFQ_EINVAL), (dict(n=BIG), E.IFQ_ERANGE), (dict(k=BIG - 7), E.IFQ_ERANGE),
    (dict(n=2 ** 30, gated=True), E.IFQ_ERANGE)])
def test_weights_refused(change, status):
    kw = dict(n=64, k=128)
    kw.update(change)
    w = ifq.w4_weights(**kw)
    assert _status(ifq.ifq_w4_bytes, w) == status
    assert _status(ifq.ifq_w4_pack, w, FAKE, FAKE, FAKE, FAKE, stream=0) == status
    f = ifq.ifq_w4_gated if w.gated else ifq.ifq_w4_matmul
    assert _status(f, ifq.w4_desc(w, 1, ifq.IFQ_BF16, 1), FAKE, FAKE, FAKE, stream=0) == status


def test_pack_refuses():
    w = ifq.w4_weights(64, 128)
    for i in range(4):
        p = [FAKE] * 4
        p[i] = None
        assert _status(ifq.ifq_w4_pack, w, *p, stream=0) == E.IFQ_EINVAL
    for p in ([FAKE + 2, FAKE, FAKE, FAKE], [FAKE, FAKE + 1, FAKE, FAKE], [FAKE, FAKE, FAKE + 1, FAKE], [FAKE, FAKE, FAKE, FAKE + 8]):
        assert _status(ifq.ifq_w4_pack, w, *p, stream=0) == E.IFQ_EALIGN


@pytest.mark.parametrize("change,status", [
    (dict(m=-1), E.IFQ_EINVAL), (dict(m=BIG), E.IFQ_ERANGE), (dict(out_dtype=0), E.IFQ_EINVAL), (dict(out_dtype=9), E.IFQ_EINVAL),
    (dict(x_stride=120), E.IFQ_EINVAL), (dict(x_stride=132), E.IFQ_EINVAL), (dict(x_stride=-8), E.IFQ_EINVAL),
    (dict(out_stride=63), E.IFQ_EINVAL), (dict(out_stride=-64), E.IFQ_EINVAL)])
def test_products_refuse(change, status):
    kw = dict(m=3, out_dtype=ifq.IFQ_BF16, act=ifq.IFQ_ACT_SILU)
    kw.update(change)
    assert _status(ifq.ifq_w4_matmul, ifq.w4_desc(ifq.w4_weights(64, 128), **kw), FAKE, FAKE, FAKE, stream=0) == status
    assert _status(ifq.ifq_w4_gated, ifq.w4_desc(ifq.w4_weights(64, 128, gated=True), **kw), FAKE, FAKE, FAKE, stream=0) == status


def test_products_refuse_pointers_and_kinds():
    d, g = ifq.w4_desc(ifq.w4_weights(64, 128), 3), ifq.w4_desc(ifq.w4_weights(64, 128, gated=True), 3, act=ifq.IFQ_ACT_GELU)
    assert _status(ifq.ifq_w4_gated, d, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    assert _status(ifq.ifq_w4_matmul, g, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    for f, e in ((ifq.ifq_w4_matmul, d), (ifq.ifq_w4_gated, g)):
        for i in range(3):
            p = [FAKE] * 3
            p[i] = None
            assert _status(f, e, *p, stream=0) == E.IFQ_EINVAL
            p[i] = FAKE + 8
            assert _status(f, e, *p, stream=0) == E.IFQ_EALIGN
    assert _status(ifq.ifq_w4_matmul, d, FAKE, FAKE, FAKE, FAKE + 4, stream=0) == E.IFQ_EALIGN
    e = ifq.w4_desc(ifq.w4_weights(64, 128), 3, residual_stride=60)
    assert _status(ifq.ifq_w4_matmul, e, FAKE, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    # out over its own residual with other rows
    e = ifq.w4_desc(ifq.w4_weights(64, 128), 3, residual_stride=72)
    assert _status(ifq.ifq_w4_matmul, e, FAKE, FAKE, 2 * FAKE, 2 * FAKE, stream=0) == E.IFQ_EINVAL
    for act in (0, 4, -1):
        e = ifq.w4_desc(ifq.w4_weights(64, 128, gated=True), 3, act=act)
        assert _status(ifq.ifq_w4_gated, e, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL
    for out in (ifq.IFQ_F16, ifq.IFQ_F32):     # a gated pair's output is of the weights' type
        e = ifq.w4_desc(ifq.w4_weights(64, 128, gated=True), 3, out, act=1)
        assert _status(ifq.ifq_w4_gated, e, FAKE, FAKE, FAKE, stream=0) == E.IFQ_EINVAL


def test_norm_refuses():
    def st(x=FAKE, residual=2 * FAKE, weight=3 * FAKE, sum=4 * FAKE, out=5 * FAKE, **kw):
        a = dict(rows=3, dim=64)
        a.update(kw)
        return _status(ifq.ifq_rms_norm, ifq.norm_desc(**a), x, residual, weight, sum, out, stream=0)

    for name in ("x", "weight", "out", "residual"):     # (a sum needs a residual)
        assert st(**{name: None}) == E.IFQ_EINVAL
    for name in ("x", "weight", "out", "residual", "sum"):
        assert st(**{name: FAKE + 8}) == E.IFQ_EALIGN
        if name != "weight":
            assert st(**{name + "_stride": 56}) == st(**{name + "_stride": 68}) == st(**{name + "_stride": -64}) == E.IFQ_EINVAL
    assert st(rows=-1) == st(dim=0) == st(dtype=ifq.IFQ_F32) == st(eps=-1e-6) == st(eps=float("nan")) == E.IFQ_EINVAL
    assert st(dim=60) == E.IFQ_ESHAPE
    assert st(dim=65544) == E.IFQ_EUNSUPPORTED
    assert st(rows=BIG) == E.IFQ_ERANGE
    assert st(sum=5 * FAKE) == E.IFQ_EINVAL             # sum and out in one buffer
    assert st(out=FAKE, x_stride=72) == st(sum=2 * FAKE, residual_stride=72) == st(sum=FAKE, sum_stride=80) == E.IFQ_EINVAL


def test_scores_refuse():
    def st(logits=FAKE, tokens=FAKE, logprobs=FAKE, lse=FAKE, entropy=FAKE, ids=FAKE, best=FAKE, **kw):
        a = dict(rows=3, vocab=100, top=4)
        a.update(kw)
        return _status(ifq.ifq_token_scores, ifq.scores_desc(**a), logits, tokens, logprobs, lse, entropy, ids, best, stream=0)

    assert st(logits=None) == st(tokens=None) == E.IFQ_EINVAL
    for name, by in (("logits", 2), ("tokens", 4), ("logprobs", 2), ("lse", 2), ("entropy", 2), ("ids", 4), ("best", 2)):
        assert st(**{name: FAKE + by}) == E.IFQ_EALIGN
    assert st(logits=FAKE + 1, dtype=ifq.IFQ_F16) == E.IFQ_EALIGN
    for kw in (dict(rows=-1), dict(vocab=0), dict(dtype=0), dict(dtype=4), dict(top=-1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(stride=99), dict(stride=-100)):
        assert st(**kw) == E.IFQ_EINVAL, kw
    assert st(top=33) == E.IFQ_EUNSUPPORTED
    assert st(vocab=3) == E.IFQ_ESHAPE
    assert st(rows=BIG) == st(vocab=BIG) == st(scale=2e30) == E.IFQ_ERANGE


def test_calls_without_rows_take_null_pointers():
    ifq.ifq_w4_matmul(ifq.w4_desc(ifq.w4_weights(64, 128), 0), None, FAKE, None, stream=0)
    ifq.ifq_w4_gated(ifq.w4_desc(ifq.w4_weights(64, 128, gated=True), 0, act=1), None, FAKE, None, stream=0)
    ifq.ifq_rms_norm(ifq.norm_desc(0, 64), None, None, None, None, None, stream=0)
    ifq.ifq_token_scores(ifq.scores_desc(0, 100, top=3), None, None, stream=0)
