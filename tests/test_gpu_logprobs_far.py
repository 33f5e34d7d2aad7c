"""Logits further apart than float32's largest number, under temperatures that bring them near."""
import numpy as np
import pytest
import torch

from test_gpu_logprobs import LARGEST, check, logits, some, tt  # noqa: F401

pytestmark = pytest.mark.gpu


# One CTA a row and clusters, of either size of CTA.
@pytest.mark.parametrize("V", [2, 300, 20000, 151936])
def test_distances_that_float32_does_not_hold(tt, V):  # noqa: F811
    T = [1e36, 1e37, 5e37, 1e38, LARGEST, np.inf, 1e30, 1.0]
    g = np.random.default_rng(V)
    x = (g.uniform(-1, 1, (len(T), V)) * LARGEST).astype(np.float32)
    x[:, 0], x[:, -1] = -LARGEST, LARGEST
    x[3, 0] = -np.inf
    tokens = np.concatenate([some(21, len(T), V, 3), np.tile([0, V - 1], (len(T), 1))], 1)
    check(tt, torch.from_numpy(x).cuda(), tokens, T=T, top=min(V, 5))


@pytest.mark.parametrize("V", [300, 151936])
def test_an_infinite_logit_among_masked_ones(tt, V):  # noqa: F811
    """Plus infinity counts as float32's largest number; masks of the lowest one."""
    x = logits(22, 4, V)
    x[:, ::3] = -LARGEST
    x[:, V // 2] = np.inf
    check(tt, x, np.tile([0, 1, V // 2, V - 1], (4, 1)), T=[1e38, 3e38, 1e20, 1.0], top=4)
