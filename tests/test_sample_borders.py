"""That the inputs of the sampler's GPU tests have one right answer: none lies next to the border of a cut or of the draw.

The kernel's weights are off by a unit of 2^-44 at most, each (test_gpu_sample_weights.py).  Among n weights a running sum and p or u times the
whole are then off by 2 n units together: an input whose top-p cut or whose draw is nearer to a border than that, or that has a weight
within a unit of min_p, might validly keep one token more or less.  Weights that are whole numbers of units (equal logits) are exact, and
so are their sums.  The same tests' functions run here with the call replaced, so their inputs are looked at as they are."""
import itertools

import numpy as np
import pytest

import step_reference as ref
import test_gpu_sample
import test_gpu_sample_draw

UNIT = 2.0 ** -44
TESTS = ["test_what_stays_lies_at_any_density", "test_settings", "test_rows_with_settings_of_their_own", "test_where_one_cta_takes_a_row", "test_clusters_of_every_size", "test_largest_vocabulary",
         "test_equal_logits_go_by_index", "test_outliers_and_masks", "test_fewer_tokens_than_top_k", "test_flat_distributions", "test_rows_without_a_token_and_what_is_not_finite"]


def distances(x, u, T, k, p, m):
    """Of top-p's cut, of min_p's and of the draw, each in what may move it; none for what is off or exact."""
    got = ref.weights(x, T)
    if got is None:
        return
    w, order = got
    n = min(k, x.size) if k > 0 else x.size
    ws = w[order][:n]
    exact = (ws / UNIT == np.rint(ws / UNIT)).all()
    if exact:
        return
    if 0 < p < 1:
        c = np.cumsum(ws.astype(np.longdouble))
        need = p * c[-1]
        j = int(np.searchsorted(c, need))
        assert j == int(np.searchsorted(np.cumsum(ws), p * ws.sum())), "the plain form's own sums are too near"
        yield float(min(c[j] - need, need - (c[j - 1] if j else -1)) / (2 * n * UNIT))
    if 0 < m <= 1:
        rest = ws[ws != 1]
        if rest.size:
            yield float(np.abs(rest - m).min() / UNIT)
    yield ref.sample(x, u, T, k, p, m)[2] / (2 * n * UNIT)


def every_call(test):
    """Calls a test once for each of its parameters."""
    sets = []
    for mark in getattr(test, "pytestmark", []):
        if mark.name == "parametrize":
            names = [s.strip() for s in mark.args[0].split(",")]
            sets.append([dict(zip(names, v if len(names) > 1 else (v,))) for v in mark.args[1]])
    for chosen in itertools.product(*sets):
        test(None, **{name: v for some in chosen for name, v in some.items()})


@pytest.mark.parametrize("name", TESTS)
def test_no_input_lies_next_to_a_border(monkeypatch, name):
    looked_at = []

    def look(_, x, u, T=None, k=None, p=None, m=None, stride=None):
        at = lambda v, r, off: off if v is None else float(np.float32(np.broadcast_to(v, len(x))[r]))  # noqa: E731
        for r in range(len(x)):
            found = list(distances(x[r], np.float32(u[r]), at(T, r, 1.0), int(at(k, r, 0)), at(p, r, 1.0), at(m, r, 0.0)))
            assert all(d > 1 for d in found), (r, found)
            looked_at.extend(found)
    module = test_gpu_sample if hasattr(test_gpu_sample, name) else test_gpu_sample_draw
    monkeypatch.setattr(module, "check", look)
    every_call(getattr(module, name))
    assert looked_at
