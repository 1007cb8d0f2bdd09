"""The oracle's 8-bit rows and head norms against torch's own conversions and hand-made values (CPU)."""
import numpy as np
import pytest
import torch

import oracle


def test_every_e4m3_byte():
    b = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    np.testing.assert_array_equal(oracle.e4m3_values(), b.view(torch.float8_e4m3fn).double().numpy())


def test_rows_round_to_the_nearest_value():
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((50, 64)) * np.exp2(rng.integers(-30, 30, size=(50, 1)))).to(torch.bfloat16)
    x[0] = 0
    x[1, 3] = float("inf")
    x[2, 5] = float("nan")
    x[3] = torch.tensor([448.0, 449.0 / 2, -448.0, 7.0] * 16, dtype=torch.bfloat16)
    x[4] = torch.tensor([450.0, 1.0, -2.0 ** -9, 2.0 ** -10] * 16, dtype=torch.bfloat16)
    q, s = oracle.q8_rows(x.double().numpy())
    assert s[0] == 7 and not (q[0] & 127).any()
    assert (s[1:3] == 255).all() and not q[1:3].any()
    assert s[3] == 127 and s[4] == 128
    for r in [0, *range(3, 50)]:
        scaled = (x[r].double() / 2.0 ** (int(s[r]) - 127)).float()
        assert scaled.abs().max() <= 448 and (s[r] == 7 or scaled.abs().max() > 224)
        assert (scaled.to(torch.float8_e4m3fn).view(torch.uint8).numpy() == q[r]).all()
    back = oracle.q8_values(q, s)
    ok = [0, *range(3, 50)]
    xv = x.double().numpy()
    # half a step of e4m3, or of its smallest values
    assert (np.abs(back[ok] - xv[ok]) <= 2.0 ** -4 * np.abs(xv[ok]) + np.exp2(s[ok].astype(float) - 127 - 10)[:, None]).all()
    assert np.isnan(back[1:3]).all()


@pytest.mark.parametrize("layer", [False, True])
def test_norms(layer):
    x = np.array([[[3.0, 4.0, 0.0, 1.0]]])
    y, hat, _ = oracle.norm_rows(x, layer, 0.5, weight=np.array([1.0, 2.0, 3.0, 4.0]), bias=np.array([0.0, 1.0, 0.0, 0.0]))
    centred = x - 2.0 if layer else x
    want = centred / np.sqrt((10 if layer else 26) / 4 + 0.5)
    np.testing.assert_allclose(hat, want, rtol=1e-15)
    np.testing.assert_allclose(y, want * [1, 2, 3, 4] + [0, 1, 0, 0], rtol=1e-15)
