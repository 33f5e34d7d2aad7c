"""The draw among more tokens than one CTA finishes: each warp puts what stays next to each other, 32 at a time are weighed, and
what is left over goes on.  Every number of leftovers comes up; a weight lost, or taken twice, moves the probability and the token."""
import numpy as np
import pytest

from test_gpu_sample import check, tt  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [6000, 40000, 151936])
@pytest.mark.parametrize("k,p", [(None, 0.9), (5000, None), (3000, 0.95)])
def test_what_stays_lies_at_any_density(tt, vocab, k, p):  # noqa: F811
    rng = np.random.default_rng(vocab)
    rows = 16
    share = np.exp(np.linspace(np.log(600 / vocab), 0, rows))  # of the tokens that may stay: from a few hundred to all
    x = np.where(rng.random((rows, vocab)) < share[:, None], rng.random((rows, vocab)), -30).astype(np.float32)
    x[:, : vocab // 3] = np.where(x[:, : vocab // 3] < 0, x[:, : vocab // 3], x[:, : vocab // 3] / 8)  # warps whose share differs
    for _ in range(3):
        check(tt, x, rng.random(rows), 1.0, k, p)
