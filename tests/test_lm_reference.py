"""The references of the decoder's operators against independent statements of the same things (CPU)."""
import numpy as np
import pytest
import torch

import lm_reference as R


@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_code_has_a_place_of_its_own(D):
    for place, first in ((R.k_place, 0), (R.v_place, 8 * D)):
        byte, shift = place(D)
        at = byte * 2 + shift // 4
        assert sorted(at.reshape(-1)) == list(range(2 * first, 2 * first + 16 * D))
        assert (shift[:, 0::2] == 0).all() and (shift[:, 1::2] == 4).all()      # the lower-numbered code first
        assert (byte[:, 0::2] == byte[:, 1::2]).all()


def test_v_words_hold_neighbouring_tokens():
    byte, _ = R.v_place(128)
    for row in range(0, 16, 2):
        for d in range(0, 128, 4):
            assert byte[row, d] % 4 == 0 and byte[row, d + 2] == byte[row, d] + 1
            assert byte[row + 1, d] == byte[row, d] + 2


def test_e4m3_values_and_rounding():
    tab = R.e4m3_table()
    ref = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(tab, ref, equal_nan=True)
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(5, 300)) * np.exp(rng.normal(0, 3, (5, 300)))).astype(np.float32)
    x[3] = 0
    q, s = R.fp8_quantise(x)
    for b in range(3):
        blk = torch.from_numpy(x[:, 128 * b:128 * b + 128])
        st = blk.abs().amax(1) * torch.tensor(1 / 448, dtype=torch.float32)
        assert np.array_equal(st.numpy(), s[b])
        y = torch.where(st[:, None] > 0, blk / st[:, None], torch.zeros_like(blk)).to(torch.float8_e4m3fn)
        # (a zero of either sign is the same value)
        assert np.array_equal(tab[y.view(torch.uint8).numpy()], tab[q[:, 128 * b:128 * b + 128]])


def test_quantised_rows_stay_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(50, 128)).astype(np.float32)
    code, scale, mn = R.quantise4(x)
    y = code * scale[:, None].astype(np.float64) + mn[:, None].astype(np.float64)
    # half a step, and what rounding scale and min to half moves the ends by
    far = np.abs(y - x).max(1)
    assert (far <= 0.5 * scale + 2.0 ** -11 * (15 * scale + np.abs(mn)) + 1e-6).all()


def test_write_and_read_round_trip():
    rng = np.random.default_rng(2)
    D, page = 64, 32
    cache = np.zeros((3, 2, page // 16, R.group_bytes(D)), np.uint8)
    k, v = rng.normal(size=(2, D)).astype(np.float32), rng.normal(size=(2, D)).astype(np.float32)
    for h in range(2):
        kc, ks, km = R.quantise4(k[h])
        vc, vs, vm = R.quantise4(v[h])
        R.write(cache, page, 2 * page + 21, h, D, (kc, ks, km), (vc, vs, vm))
        (kv, _, _), (vv, _, _) = R.read(cache, page, [2 * page + 21], D)
        assert np.array_equal(kv[0, h], kc * float(ks) + float(km)) and np.array_equal(vv[0, h], vc * float(vs) + float(vm))
    assert cache[:2].sum() == 0
