"""Pins of the 8-bit cache's oracle that need no GPU: its rounding against torch's casts, its scales against their definition,
its attention against torch's softmax, its selection against a sort."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_cache as oracle


def test_nearest_codes():
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** -7, np.arange(-448, 449) / 2.0, np.arange(-64, 65) * 2.0 ** -10])
    want = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.nearest(y.astype(np.float32).astype(np.float64), "e4m3"), want)
    assert oracle.nearest(np.array([0.5, 1.5, -2.5, 126.5]), "i8").tolist() == [0, 2, -2, 126]


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_scales(code):
    limit = oracle.LIMIT[code]
    for most in [limit, np.nextafter(limit, 1e9), 1.0, 3e38, 1e-20, limit * 2.0 ** -77, limit * 1.0001 * 2.0 ** -77]:
        s = oracle.scale_for(most, code)
        assert math.frexp(s)[0] == 0.5 and limit * s / 2 < most <= limit * s
    assert oracle.scale_for(0.0, code) == 2.0 ** -100 == oracle.scale_for(1e-44, code)
    assert math.isnan(oracle.scale_for(math.inf, code)) and math.isnan(oracle.scale_for(math.nan, code))


def test_attention_is_a_masked_softmax():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((1, 4, 5, 8)), rng.standard_normal((1, 2, 12, 8)), rng.standard_normal((1, 2, 12, 8))
    out, lse, w, _, _, _ = oracle.attend(q, k, v, [9], [4], 0.3, True)
    z = torch.from_numpy(0.3 * np.einsum("htd,hnd->htn", q[0, :, :4], k[0].repeat(2, 0)[:, :9]))
    z = z + torch.full((4, 9), -math.inf, dtype=torch.float64).triu(9 - 4 + 1)
    p = z.softmax(2)
    assert np.allclose(out[0, :, :4], (p @ torch.from_numpy(v[0].repeat(2, 0)[:, :9])).numpy()) and not out[0, :, 4].any()
    assert np.allclose(lse[0, :, :4], z.logsumexp(2).numpy()) and np.isneginf(lse[0, :, 4]).all()
    assert np.allclose(w[0, :, :9], p.view(2, 2, 4, 9).sum((1, 2)).numpy()) and not w[0, :, 9:].any()


def test_selection():
    w = np.array([0.0, 5.0, 1.0, 1.0, -0.0, np.nan, 1.0, 9.0], np.float32)
    assert oracle.select(w, 8, 4, 1, 1).tolist() == [0, 1, 5, 7]
    assert oracle.select(w, 8, 5, 1, 1).tolist() == [0, 1, 2, 5, 7]
    assert oracle.select(w, 8, 2, 1, 1).tolist() == [0, 7] and oracle.select(w, 3, 4, 1, 1).tolist() == [0, 1, 2]


def test_a_block_grows():
    codes, scale = np.zeros((1, 1, 32, 64)), np.ones((1, 1, 1))
    oracle.append(codes, scale, np.full((1, 1, 1, 64), 3.0), [0], [1], "i8")
    assert scale[0, 0, 0] == 2.0 ** -5 and codes[0, 0, 0, 0] == 96
    oracle.append(codes, scale, np.full((1, 1, 2, 64), 10.0), [1], [1], "i8")
    assert scale[0, 0, 0] == 2.0 ** -3 and codes[0, 0, :3, 0].tolist() == [24, 80, 0]
