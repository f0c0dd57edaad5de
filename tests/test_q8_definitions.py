"""The definitions that the GPU tests of the cache in eight bits use, against torch and the
bounds that the header states."""
import numpy as np
import pytest
import torch

import q8_testlib as q8


def test_e4m3_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-14, 8.8, 5000), [0.0, 2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875, 463.9]])
    x = x.astype(np.float32)
    assert np.array_equal(q8.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_rows_are_within_half_a_step(fmt):
    g = torch.Generator().manual_seed(1)
    for scale in (1e-42, 1e-30, 1.0, 3e36):
        y = (torch.randn((200, 128), generator=g) * scale).clamp(-3.4e38, 3.4e38).numpy()
        c, z = q8.quantised(y, fmt)
        assert np.all(np.abs(c) <= q8.TOP[fmt]) and np.all(z >= q8.TINIEST)
        v = c * z.astype(np.float64)[:, None]
        # (the quotient is rounded to float32 first: 2^-24 of it)
        assert np.all(np.abs(v - y) <= q8.half_step(y, z.astype(np.float64)[:, None], fmt) + 2.0 ** -24 * np.abs(y) * (1 + 2 ** -20))
        assert np.array_equal(q8.numbers(q8.codes(c, fmt)), c)
    y = np.ones((3, 64), np.float32)
    y[0, 5], y[1, 6] = np.nan, -np.inf
    c, z = q8.quantised(y, fmt)
    assert np.isnan(z[:2]).all() and (c[:2] == 0).all() and (c[2] == q8.TOP[fmt]).all()
