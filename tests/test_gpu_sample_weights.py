"""The sampler's weights are off by no more than one unit of 2^-44: seen through min_p, whose border is a float32 m, a whole
multiple of 2^-24.

Each case is a row [0, d] with a temperature T at which w = exp(d / T) lies within 1.2 units of m.  Where w >= m, the weight that is used is
a whole number of units that is not below m either (the next one below is more than one unit off), so the second token stays; where
w < m by more than one unit, the weight that is used is below m, so it goes.  With u next to one the last token that stays is taken.
The exponent 64 log2(e) d / T lies next to half a whole number, where the table's entries meet and a short series is
farthest off: in the first block of a power of two, whose weights are largest, an error shows most."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

# (T, d, m), found by a search over float32 numbers; where w lies is computed below
NEAR = [
    (0.408882618, -0.00222081109, 0.994583309), (1.72705162, -0.00942142401, 0.994559646), (3.3221271, -0.0180745106, 0.99457413),
    (2.68950415, -0.0146896932, 0.99455303), (2.81430626, -0.0153006753, 0.994578004), (2.11777306, -0.0114810551, 0.994593382),
    (3.30783153, -0.0180573948, 0.994555891), (2.73481703, -0.0148644149, 0.994579494),
    (2.17607403, -0.0117334826, 0.994622469), (0.363149643, -0.00195977208, 0.994617939), (1.08105361, -0.00584009988, 0.994612336),
    (1.12058806, -0.00602332084, 0.994639277), (1.50004244, -0.00806806609, 0.99463588), (3.56525111, -0.0192855168, 0.994605303),
    (1.53432357, -0.00830274448, 0.994603276), (3.70999408, -0.020153407, 0.994582534),
]


def units_above(T, d, m):
    """How many units of 2^-44 exp(d / T) lies above m, from the float32 numbers, in 50 digits."""
    getcontext().prec = 50
    T, d, m = (Decimal(float(np.float32(v))) for v in (T, d, m))
    return float(((d / T).exp() - m) * 2 ** 44)


@pytest.mark.parametrize("vocab", [2, 40000])  # one CTA, a cluster
@pytest.mark.parametrize("top_k", [0, 2, 200])  # the draw over all, few candidates, the first found by a histogram
def test_a_weight_is_off_by_no_more_than_its_unit(vocab, top_k):
    from paper_2609_35465_b200 import tetra
    n = len(NEAR)
    off = np.array([units_above(*c) for c in NEAR])
    stays, goes = off >= 0, off < -1
    assert (stays | goes).all() and stays.any() and goes.any() and np.abs(off).max() < 1.2
    x = torch.full((n, vocab), -float("inf"), device="cuda")
    x[:, 0] = 0
    x[:, vocab - 1] = torch.tensor([c[1] for c in NEAR], device="cuda")
    column = lambda i: torch.tensor([c[i] for c in NEAR], device="cuda")  # noqa: E731
    tokens = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    k = torch.full((n,), top_k, dtype=torch.int32, device="cuda")
    tetra.tetra_sample(x, torch.full((n,), 0.999, device="cuda"), tokens, temperature=column(0), min_p=column(2), top_k=k)
    assert tokens.tolist() == np.where(stays, vocab - 1, 0).tolist()
