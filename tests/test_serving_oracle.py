"""Pins of the fp64 oracles of the 8-bit matrices and of sampling."""

import numpy as np
import pytest
import torch

from oracle import sampling as S
from oracle import scaled as Q

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_every_code_decodes_and_rounds_to_itself(code):
    bits = np.arange(256, dtype=np.uint8)
    v = torch.from_numpy(bits).view(TORCH[code]).double().numpy()
    fine = np.isfinite(v)
    np.testing.assert_array_equal(Q.decode(bits[fine], code), v[fine])
    np.testing.assert_array_equal(Q.encode(v[fine], code), bits[fine])
    np.testing.assert_array_equal(Q.round_to_code(v[fine], code), v[fine])


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_rounding_agrees_with_the_conversion_of_torch(code):
    x = np.random.default_rng(0).standard_normal(20000).astype(np.float32) * np.float32(10) ** np.linspace(-9, 2, 20000, dtype=np.float32)
    x = np.clip(x, -Q.LARGEST[code], Q.LARGEST[code])
    ties = np.array([0.0, 17.0, 19.0, 1.0625, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -17, 3 * 2.0 ** -17], dtype=np.float32)
    x = np.concatenate([x, ties, -ties])
    np.testing.assert_array_equal(Q.round_to_code(x, code), torch.from_numpy(x).to(TORCH[code]).double().numpy())


def test_blocks_and_scales_by_hand():
    x = np.zeros((130, 129), dtype=np.float32)
    x[0, 0], x[129, 0], x[5, 128] = 448.0, -7.0, 2.0
    q, s = Q.quantize(x, 128, "e4m3")
    assert s.shape == (2, 2)
    np.testing.assert_array_equal(s, np.array([[1.0, 7.0 / 448.0], [2.0 / 448.0, 2.0 ** -100]], dtype=np.float32))
    assert q[0, 0] == 448 and q[129, 0] == -448 and q[5, 128] == 448
    np.testing.assert_allclose(Q.values(q, s, 128), x, rtol=2.0 ** -23)
    q, s = Q.quantize(x, 1, "e5m2")
    assert s.shape == (2, 130) and q[5, 128] == 57344


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    assert [S.sample(x, u)[0] for u in (0.0, 0.05, 0.11, 0.49, 0.51, 0.71, 0.999)] == [0, 0, 1, 1, 2, 3, 3]
    np.testing.assert_allclose(S.kept_mass(x, top_k=2), [0, 1, 0, 0.75])
    np.testing.assert_allclose(S.kept_mass(x, top_p=0.69), [0, 1, 0, 0.75])
    np.testing.assert_allclose(S.kept_mass(x, top_p=0.71), [0, 1, 0.5, 0.75])
    np.testing.assert_allclose(S.kept_mass(x, top_k=3, top_p=0.77), [0, 1, 0, 0.75])      # of 0.9: 0.4 + 0.3 = 0.7 = 0.778 of it
    np.testing.assert_allclose(S.kept_mass(x, min_p=0.6), [0, 1, 0, 0.75])
    np.testing.assert_allclose(S.kept_mass(x, temperature=0.5), [0.0625, 1, 0.25, 0.5625])
    np.testing.assert_allclose(S.kept_mass(x, temperature=0.0), [0, 1, 0, 0])
    np.testing.assert_allclose(S.kept_mass(x, allowed=np.array([1, 0, 1, 1], bool), top_k=1), [0, 0, 0, 1])
    assert S.sample(x, 1.0)[0] == 3 and S.sample(x, 0.5, top_p=0.0)[0] == 1
    assert abs(S.sample(x, 0.5)[2] - 0.4) < 1e-12
    ties = np.zeros(5)
    np.testing.assert_allclose(S.kept_mass(ties, top_k=2), [1, 1, 0, 0, 0])               # equal logits: the lower ids
    np.testing.assert_allclose(S.kept_mass(ties, top_p=0.5), [1, 1, 1, 0, 0])
    for bad in ([np.nan, 1.0], [np.inf, 1.0], [-np.inf, -np.inf]):
        assert S.sample(np.array(bad), 0.5)[:3] == (-1, 0.0, 0.0)
    assert S.sample(x, 0.5, temperature=np.nan)[0] == -1 and S.sample(x, np.nan)[0] == -1
