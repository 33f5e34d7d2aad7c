"""Norms of queries of any size that float32 holds, by either kernel: rows that are large, tiny or zero, an eps below float32's normal numbers."""
import numpy as np
import pytest
import torch

from test_gpu_kv import INV, Step, dev, i32
from test_gpu_kv_append_at import plain_rows, tt  # noqa: F401

pytestmark = pytest.mark.gpu

# A row's size, and eps.
SIZES = [(1e19, 1e-6), (1.9e18, 1e-6), (3e37, 1e-6), (1e25, 0.0), (1e-25, 0.0), (1e-19, 0.0), (1e-37, 0.0), (1e-25, 1e-50), (1e-25, 1e-60), (1e-12, 1e-24), (1e-13, 1e-6), (1.0, 0.0), (1.0, 1e30),
         (1e30, 1e60), (1e10, 1e38)]


@pytest.mark.parametrize("rows", [[3, 1], [90, 40]])  # a row a CTA, a block a CTA
@pytest.mark.parametrize("D,heads,offset", [(64, 9, 0), (128, 4, 0), (128, 4, 1), (256, 7, 0)])
def test_norms_of_rows_of_any_size(tt, D, heads, offset, rows):  # noqa: F811
    H = 1
    st = Step(601, D, H, 16, [5, 0], rows)
    n, rng = st.total, st.rng
    positions, axis = rng.integers(-1000, 1000, (n, 3)), rng.integers(0, 3, D // 2).astype(np.uint8)
    for size, eps in SIZES:
        x = rng.standard_normal((n, heads + 2 * H, D))
        x = (x / np.abs(x).max() * size * 2.0 ** -rng.integers(0, 3, (n, heads + 2 * H, 1))).astype(np.float32)
        weight = (1 + 0.3 * rng.standard_normal(D)).astype(np.float32)
        x[0, 0] = 0 if eps else x[0, 0]             # zeros stay zeros
        x[1, 1, :D // 2] *= np.float32(2.0 ** -20)  # halves of very different size
        flat = torch.zeros((n, (heads + 2 * H) * D + offset), device="cuda")
        flat[:, offset:] = dev(x).flatten(1)
        d = flat[:, offset:].unflatten(1, (heads + 2 * H, D))
        out = torch.full((n, heads, D), 7.5, dtype=torch.float16, device="cuda")
        tt.tetra_kv_append_at(d[:, :heads], d[:, heads:heads + H], d[:, heads + H:], *st.args(), i32(positions), dev(axis), out, dev(INV[D]), q_weight=dev(weight), eps=eps)
        # float32's least normal number is the least that counts: smaller elements of a row are zero
        seen = np.where(np.abs(x) < 2.0 ** -126, 0, x).astype(np.float64)
        with np.errstate(invalid="ignore"):
            want = plain_rows(seen[:, :heads], weight, positions, axis, INV[D], eps)
        a, b = np.split(want, 2, -1)
        pair = np.sqrt(2) * np.concatenate([np.hypot(a, b)] * 2, -1)  # |a| + |b| at most
        have = out.cpu().numpy().astype(np.float64)
        # as in test_gpu_kv_append_at: one rounding to float16, and 2^-20 of |a| + |b| for what is in 32 bits
        off = np.abs(have - want) - (2.0 ** -11 * np.abs(want) + 2.0 ** -20 * pair + 2.0 ** -25)
        none = np.isnan(want)  # a row of zeros without an eps
        assert np.array_equal(np.isnan(have), none) and not (none.any() and eps)
        assert (off[~none] <= 0).all(), (size, eps, have[off > 0][:4], want[off > 0][:4])


@pytest.mark.parametrize("rows", [[3, 1], [90, 40]])
def test_weights_of_any_size(tt, rows):  # noqa: F811
    """A large element that a small weight brings down beside small ones that a large weight brings up."""
    D, heads, H = 128, 4, 1
    st = Step(602, D, H, 16, [5, 0], rows)
    n, rng = st.total, st.rng
    x = (2.0 ** -60 * rng.standard_normal((n, heads + 2 * H, D))).astype(np.float32)
    x[..., 3] = 2.0 ** 50
    weight = np.full(D, 2.0 ** 105, np.float32)
    weight[3] = 2.0 ** -3
    positions, axis = rng.integers(-1000, 1000, (n, 3)), rng.integers(0, 3, D // 2).astype(np.uint8)
    d = dev(x)
    out = torch.zeros((n, heads, D), dtype=torch.float16, device="cuda")
    tt.tetra_kv_append_at(d[:, :heads], d[:, heads:heads + H], d[:, heads + H:], *st.args(), i32(positions), dev(axis), out, dev(INV[D]), q_weight=dev(weight))
    want = plain_rows(x[:, :heads], weight, positions, axis, INV[D])
    a, b = np.split(want, 2, -1)
    pair = np.sqrt(2) * np.concatenate([np.hypot(a, b)] * 2, -1)
    assert (np.abs(out.cpu().numpy() - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -20 * pair + 2.0 ** -25).all()
