"""The plain references against hand-made cases (no GPU)."""
import numpy as np
import pytest
import torch

import layer_reference as R


def test_rounding():
    x = np.concatenate([np.random.default_rng(0).normal(size=4000) * 10.0 ** np.random.default_rng(1).integers(-30, 30, 4000),
                        [1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 0.0, -0.0, np.inf, -np.inf]]).astype(np.float32)
    t = torch.from_numpy(x)
    assert np.array_equal(R.round_to(x, "bf16"), t.bfloat16().double().numpy())
    assert np.array_equal(R.round_to(x, "f16"), t.half().double().numpy())
    assert np.isnan(R.round_to(np.nan, "bf16"))


def test_weights_by_hand():
    codes = np.array([[0x21, 0x43] + [0] * 14 + [0xF0]], np.uint8)                   # columns 1, 2, 3, 4, 0 ..., 0, 15
    w = R.weights(codes, np.array([[0.5, 2.0]]), np.array([[-1.0, 100.0]]), 32, "bf16")
    assert w[0, :5].tolist() == [-0.5, 0.0, 0.5, 1.0, -1.0]
    assert w[0, 32:].tolist() == [100.0, 130.0]
    assert R.weights(codes, np.array([[0.5, 2.0]]), np.array([[-1.0, 257.0]]), 32, "bf16")[0, 33] == 288.0   # 287 is between


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_activations(name):
    a = np.linspace(-9, 9, 41)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[name]
    np.testing.assert_allclose(R.act(name, a), f(torch.from_numpy(a)).numpy(), rtol=1e-6, atol=1e-12)


def test_scores_by_hand():
    x = np.array([[0.0, np.log(3.0), -np.inf, np.log(3.0)], [-np.inf] * 4, [0.0, np.nan, 1.0, np.inf], [2.0, np.inf, 1.0, 1.0]])
    s = R.scores(x, [2, 0, 0, 9], 1.0, 3)
    np.testing.assert_allclose(s["lse"][0], np.log(7.0))
    np.testing.assert_allclose(s["entropy"][0], -(6 / 7 * np.log(3 / 7) + 1 / 7 * np.log(1 / 7)))
    assert s["top_ids"].tolist() == [[1, 3, 0], [0, 1, 2], [1, 3, 2], [1, 0, 2]]
    assert s["logprobs"][0] == -np.inf and s["lse"][1] == -np.inf and s["entropy"][1] == 0
    assert np.isnan(s["lse"][2]) and s["lse"][3] == np.inf and np.isnan(s["entropy"][3]) and np.isnan(s["logprobs"][3])


def test_norm_by_hand():
    out, h = R.rms_norm(np.array([[3.0, 4.0]]), np.array([[0.0, 2.0 ** -9]]), np.array([1.0, 2.0]), 0.0, "bf16")
    assert h.tolist() == [[3.0, 4.0]]
    np.testing.assert_allclose(out, [[3 / 12.5 ** 0.5, 8 / 12.5 ** 0.5]])
