"""The norm between the blocks.  The sum is exact to its definition; out is off by its rounding and by 2^-18 of the value
(the sum of squares in single precision: chains of at most 64 + 10 additions of 2^-24 each, half of that after the root;
four more roundings and the root's 2^-22)."""
import numpy as np
import pytest
import torch

import layer_reference as R
from paper_1911_08076_gb300 import ifq

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = {"f16": (ifq.IFQ_F16, torch.float16), "bf16": (ifq.IFQ_BF16, torch.bfloat16)}


def rows_of(a, dtype, pad=0):
    t = torch.full((a.shape[0], a.shape[1] + pad), float("nan"), device=DEV, dtype=TYPES[dtype][1])
    t[:, :a.shape[1]] = torch.from_numpy(a.astype(np.float32)).to(DEV).to(TYPES[dtype][1])
    return t


def smallest(dtype):
    return {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}[dtype]


def check(x, r, w, eps, dtype, pads=(0, 0, 0, 0), seed=0):
    rows, dim = x.shape
    xd, rd = rows_of(x, dtype, pads[0]), None if r is None else rows_of(r, dtype, pads[1])
    wd = rows_of(w[None], dtype)
    sd = None if r is None else torch.full((rows + 1, dim + pads[2]), 7.0, device=DEV, dtype=TYPES[dtype][1])
    od = torch.full((rows + 1, dim + pads[3]), 7.0, device=DEV, dtype=TYPES[dtype][1])
    d = ifq.norm_desc(rows, dim, TYPES[dtype][0], eps, dim + pads[0], dim + pads[1], dim + pads[2], dim + pads[3])
    ifq.ifq_rms_norm(d, xd, rd, wd, sd, od)
    out, h = R.rms_norm(x, r, w, float(np.float32(eps)), dtype)
    got = od[:rows, :dim].double().cpu().numpy()
    assert (od[rows:] == 7).all() and (od[:, dim:] == 7).all()
    if r is not None:
        assert np.array_equal(sd[:rows, :dim].double().cpu().numpy(), h)
        assert (sd[rows:] == 7).all() and (sd[:, dim:] == 7).all()
    err = np.abs(got - out)
    tol = np.abs(out) * (R.half_step(dtype) + 2.0 ** -18) + smallest(dtype)
    assert (err <= tol).all(), np.max(err / tol)


@pytest.mark.parametrize("rows,dim", [(1, 8), (1, 4096), (1, 8200), (3, 248), (2, 32768), (1, 65536), (5, 40000), (7, 1032),
                                      (400, 2048), (1000, 136), (333, 5000), (310, 65536), (2, 16384), (3, 16392), (400, 16384), (305, 32768), (2, 32776), (1003, 8), (2001, 1024), (17, 256), (3000, 1032)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("residual", [True, False])
def test_values(rows, dim, dtype, residual):
    rng = np.random.default_rng([rows, dim])
    x = R.round_to(rng.normal(size=(rows, dim)), dtype)
    r = R.round_to(rng.normal(size=(rows, dim)) * np.where(rng.random(dim) < 0.02, 30, 2), dtype) if residual else None
    check(x, r, R.round_to(1 + 0.2 * rng.normal(size=dim), dtype), 1e-5, dtype,
          (8, 16, 24, 8) if rows % 2 else (0, 0, 0, 0))


@pytest.mark.parametrize("rows", [2, 400])
@pytest.mark.parametrize("scale,eps", [(2.0 ** 100, 1e-5), (2.0 ** 126, 0.0), (2.0 ** -80, 0.0), (2.0 ** -120, 0.0), (2.0 ** -80, 1e-6),
                                       (1.0, 1e4), (0.0, 1e-5)])
def test_far_ends_of_bfloat16(rows, scale, eps):
    rng = np.random.default_rng(1)
    x = R.round_to(rng.uniform(0.5, 1.9, size=(rows, 512)) * scale, "bf16")
    check(x, None, R.round_to(rng.normal(size=512), "bf16"), eps, "bf16")


def test_rows_of_zeros_without_eps_and_what_is_not_finite():
    x = np.ones((6, 64))
    x[0], x[2, 3], x[4, 9] = 0, np.inf, np.nan
    xd, w, out = rows_of(x, "bf16"), rows_of(np.ones((1, 64)), "bf16"), torch.empty(6, 64, dtype=torch.bfloat16, device=DEV)
    ifq.ifq_rms_norm(ifq.norm_desc(6, 64, eps=0.0), xd, None, w, None, out)
    got = out.double().cpu().numpy()
    assert np.isnan(got[0]).all() and np.isnan(got[4]).all()           # 0 / 0
    assert np.isnan(got[2, 3]) and (np.delete(got[2], 3) == 0).all()   # inf / inf, 1 / inf
    assert (got[[1, 3, 5]] == 1).all()


@pytest.mark.parametrize("rows", [3, 500])
def test_in_place(rows):
    rng = np.random.default_rng(5)
    x, r = (rows_of(rng.normal(size=(rows, 264)), "bf16") for _ in range(2))
    w = rows_of(rng.normal(size=(1, 264)), "bf16")
    d = ifq.norm_desc(rows, 264)
    s, o = torch.empty_like(x), torch.empty_like(x)
    ifq.ifq_rms_norm(d, x, r, w, s, o)
    for sum_at, out_at in (("r", "x"), ("x", "r"), ("r", None), (None, "r"), (None, "x")):
        t = {"x": x.clone(), "r": r.clone()}
        sd = t[sum_at] if sum_at else None
        od = t[out_at] if out_at else torch.empty_like(x)
        ifq.ifq_rms_norm(d, t["x"], t["r"], w, sd, od)
        assert torch.equal(od, o) and (sd is None or torch.equal(sd, s))
    t = x.clone()
    p = torch.empty_like(x)
    ifq.ifq_rms_norm(d, x, None, w, None, p)
    ifq.ifq_rms_norm(d, t, None, w, None, t)
    assert torch.equal(t, p)
