"""Rows at given positions of several axes on the GPU against the plain form in 64 bits: codes and scales are equal; queries are rounded
once, and of many rows a sequence made in 32 bits from there on where the sines are known."""
import numpy as np
import pytest
import torch

import step_reference as ref
from test_gpu_kv import INV, Step, dev, i32, same_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def plain_rows(x, weight, positions, axis, inv_freq, eps=1e-6):
    """Norm and rotation of rows [rows, heads, D], float64."""
    at = np.where(axis < positions.shape[1], positions[:, np.minimum(axis, positions.shape[1] - 1)], 0).astype(np.float64) * inv_freq
    return np.stack([ref.turned(x[r], weight, at[r], 1, eps) for r in range(len(x))]) if len(x) else x.astype(np.float64)


def append_both(tt, st, heads, axes=3, dtype=np.float32, norm=True, spread=1.0, edit=None, far=10000, q=True, sliced=True, stride=0):
    rng, n, D, H = st.rng, st.total, st.D, st.H
    x = (rng.standard_normal((n, heads + 2 * H, D)) * np.exp(spread * rng.standard_normal((n, heads + 2 * H, 1)))).astype(dtype)
    if edit:
        edit(x)
    parts = x[:, :heads], x[:, heads:heads + H], x[:, heads + H:]
    w = [1 + 0.3 * rng.standard_normal(D).astype(np.float32) if norm else None for _ in range(2)]
    positions = rng.integers(-far, far, (n, axes + stride))
    axis = rng.integers(0, axes, D // 2).astype(np.uint8)
    used = positions[:, :axes]
    plain = st.plain()
    with np.errstate(invalid="ignore"):
        turned = [plain_rows(parts[i], w[i], used, axis, INV[D]) for i in range(2)]
    plain.append(turned[0], turned[1], parts[2], st.table, st.starts, st.before)
    want = np.full(turned[0].shape, np.nan)
    for s in range(len(st.before)):
        want[st.starts[s]:st.starts[s + 1]] = turned[0][st.starts[s]:st.starts[s + 1]]
    d = dev(x)
    given = [d[:, :heads], d[:, heads:heads + H], d[:, heads + H:]]
    if not sliced:
        given = [p.contiguous() for p in given]
    out = torch.full((n, heads, D), 7.5, dtype=torch.float16, device="cuda") if q else None
    got = tt.tetra_kv_append_at(given[0] if q else None, *given[1:], *st.args(), i32(positions)[:, :axes], dev(axis), out, dev(INV[D]), q_weight=dev(w[0]) if norm else None,
                                k_weight=dev(w[1]) if norm else None, eps=1e-6)
    assert got is out
    if q:
        o = out.cpu().numpy().astype(np.float64)
        nobody = np.isnan(want).all((1, 2))
        nobody[:int(st.starts[-1])] = False
        assert (o[nobody] == 7.5).all()
        ok, have = want[~nobody], o[~nobody]
        a, b = np.split(ok, 2, -1)
        size = np.sqrt(2) * np.concatenate([np.hypot(a, b)] * 2, -1)  # |a| + |b| of a pair at most
        fine = np.abs(ok) + 2.0 ** -20 * size < 65504
        # Rounded once: half a step, relative 2^-11, or 2^-25 below the least normal number.  In 32 bits: the sum of squares is off by 13 2^-24 at most, its
        # root by half of that, the reciprocal root by 2^-22, two products, the sines and the rotation by 7 2^-24: 2^-20 of |a| + |b| together.
        assert (np.abs(have - ok)[fine] <= 2.0 ** -11 * np.abs(ok[fine]) + 2.0 ** -20 * size[fine] + 2.0 ** -25).all()
    same_cache(st, plain)
    return plain


@pytest.mark.parametrize("D,H,heads,P,before,rows", [
    (128, 8, 32, 64, [700], [1]),
    (128, 8, 40, 32, [0, 15, 16, 31, 32, 100], [1] * 6),
    (64, 2, 16, 16, [0, 3, 16, 47], [16, 14, 1, 2]),
    (256, 1, 7, 48, [5, 40], [50, 9]),
    (128, 3, 3, 128, [127, 0, 255], [2, 0, 33]),
    (128, 2, 24, 16, [11], [160]),                 # many rows: by blocks
    (64, 1, 9, 32, [3, 16, 0], [70, 64, 129]),
    (256, 2, 2, 16, [31, 15], [40, 200]),
    (128, 4, 4, 64, [37, 0, 5], [100, 0, 331]),
    (64, 1, 20, 16, [1], [47]),
])
@pytest.mark.parametrize("axes,dtype,norm", [(3, np.float32, True), (1, np.float16, False), (8, np.float32, False), (2, np.float16, True)])
def test_append_at(tt, D, H, heads, P, before, rows, axes, dtype, norm):
    append_both(tt, Step(201 + D + H + heads, D, H, P, before, rows, spare=2, gap=3), heads, axes, dtype, norm, stride=axes % 3)


def test_rows_that_are_not_slices_and_no_queries(tt):
    append_both(tt, Step(202, 128, 2, 16, [5, 0], [90, 70]), 6, sliced=False)
    append_both(tt, Step(203, 128, 2, 16, [5, 0], [90, 70]), 6, q=False)
    append_both(tt, Step(204, 64, 2, 16, [5, 0], [1, 2]), 6, q=False)


def test_odd_offsets_of_queries(tt):
    """Rows whose queries are not aligned for more than one element at a time."""
    for dtype in (torch.float16, torch.float32):
        D, H, heads, n = 128, 1, 2, 80
        st = Step(205, D, H, 16, [3], [n])
        wide = torch.randn((n, (heads + 2 * H) * D + 1), device="cuda").to(dtype)
        x = wide[:, 1:].unflatten(1, (heads + 2 * H, D))
        pos, axis = i32(np.arange(3 * n).reshape(n, 3)), torch.arange(D // 2, device="cuda").remainder(3).byte()
        outs, caches = [], []
        for t in (x, x.contiguous()):
            st.cache.copy_(dev(st.raw))
            outs.append(tt.tetra_kv_append_at(t[:, :heads], t[:, heads:heads + H], t[:, heads + H:], *st.args(), pos, axis, torch.empty((n, heads, D), dtype=torch.float16, device="cuda"), dev(INV[D])))
            caches.append(st.cache.clone())
        assert torch.equal(*outs) and torch.equal(*caches)


def test_one_axis_at_the_slots_is_append(tt):
    """The same positions on all axes: the cache is tetra_kv_append's, whatever the cut into calls."""
    D, H, heads = 128, 2, 8
    for before, rows in (([10, 0], [1, 3]), ([10, 0], [200, 90])):
        st = Step(206, D, H, 16, before, rows)
        n = st.total
        x = torch.randn((n, heads + 2 * H, D), device="cuda")
        parts = x[:, :heads], x[:, heads:heads + H], x[:, heads + H:]
        at = np.concatenate([np.arange(b, b + r) for b, r in zip(before, rows)])
        a = tt.tetra_kv_append(*parts, *st.args(), torch.empty((n, heads, D), dtype=torch.float16, device="cuda"), inv_freq=dev(INV[D]))
        first = st.cache.clone()
        st.cache.copy_(dev(st.raw))
        b = tt.tetra_kv_append_at(*parts, *st.args(), i32(np.stack([at] * 3, 1)), torch.arange(D // 2, device="cuda").remainder(3).byte(), torch.empty_like(a), dev(INV[D]))
        assert torch.equal(first, st.cache)
        assert (a.float() - b.float()).abs().max() <= 2.0 ** -10 * a.float().abs().max()


def test_far_and_negative_positions_and_axes_that_are_not_there(tt):
    """Angles of 2^31 turns keep their fraction (float64: 2^31 2^-53 of a turn); an axis beyond the last does not turn."""
    for rows in ([3], [60]):
        st = Step(207, 64, 1, 16, [0], rows)
        D, n = 64, st.total
        pos = np.array([[2 ** 31 - 1, -2 ** 31, 123456789]] * n)
        axis = np.arange(D // 2) % 5  # 3 and 4 are not there
        x = st.rng.standard_normal((n, 3, D)).astype(np.float32)
        out = tt.tetra_kv_append_at(dev(x[:, :1]), dev(x[:, 1:2]), dev(x[:, 2:]), *st.args(), i32(pos), dev(axis.astype(np.uint8)), torch.empty((n, 1, D), dtype=torch.float16, device="cuda"), dev(INV[D]))
        want = plain_rows(x[:, :1], None, pos, axis, INV[D])
        # the product with inv_freq and the one with 1 / 2 pi are rounded: 2^31 2^-52 2 pi of the angle, 2^-18.3
        assert np.abs(out.cpu().numpy() - want).max() <= (2.0 ** -11 + 2.0 ** -18 + 2.0 ** -19) * np.abs(x).max() * np.sqrt(2)


def test_what_is_not_finite_and_zeros(tt):
    def edit(x):
        x[0] = 0
        x[3, 2, 7] = np.nan     # a key of head 0 (behind two query heads)
        x[20, 5, 3] = np.inf    # a value of head 1 in a whole block
        x[40, 3, 1] = -np.inf
        x[60] *= 1e30
    for rows in ([70], [17, 17, 36]):
        st = Step(208, 64, 2, 16, [5] + [0] * (len(rows) - 1), rows)
        plain = append_both(tt, st, 2, norm=False, edit=edit)
        assert np.isnan(plain.scales).any()


def test_slots_that_are_not_there(tt):
    for rows in ([2, 5, 1, 1, 1], [40, 33, 50, 35, 40]):
        st = Step(209, 128, 2, 16, [-3, 30, 2 ** 31 - 3, 40, 17], rows, width=2)
        st.table[3] = [-1, -2 ** 31]
        st.table[4] = [0, st.pages]
        st.d_table = i32(st.table)
        append_both(tt, st, 4)


def test_ranges_of_rows_that_make_no_sense_have_no_rows(tt):
    for n in (4, 100):
        st = Step(210, 64, 1, 16, [0] * 4, [n // 4] * 4)
        x = torch.randn((n, 4, 64), device="cuda")
        pos, axis = i32(np.zeros((n, 1))), torch.zeros(32, dtype=torch.uint8, device="cuda")
        for starts in ([-5, -1, -1, -1, -1], [n + 1] * 5, [0, 0, 0, 0, 0], [0, n + 7, n + 9, n + 9, n + 9]):
            out = torch.full((n, 2, 64), 7.5, dtype=torch.float16, device="cuda")
            tt.tetra_kv_append_at(x[:, :2], x[:, 2:3], x[:, 3:], st.cache, st.d_table, i32(starts), st.d_lengths, pos, axis, out, dev(INV[64]))
            assert (out == 7.5).all() and torch.equal(st.cache, dev(st.raw))


def test_many_sequences_by_blocks(tt):
    rng = np.random.default_rng(211)
    append_both(tt, Step(211, 64, 1, 16, rng.integers(0, 40, 90).tolist(), rng.integers(20, 90, 90).tolist()), 2, sliced=False)


def test_reading_many_rows(tt):
    """tetra_kv_read by blocks: odd beginnings and ends, sequences without rows, places that are not there."""
    st = Step(212, 128, 3, 32, [0] * 5, [200, 0, 37, 331, 64], spare=2)
    st.table[3, 2] = -1
    st.d_table = i32(st.table)
    for before in ([0] * 5, [3, 0, 16, 40, 15]):
        k, v = (torch.full((st.total, 3, 128), 7.5, dtype=torch.float16, device="cuda") for _ in range(2))
        tt.tetra_kv_read(st.cache, st.d_table, st.d_starts, i32(before), k, v)
        plain = st.plain()
        for s, (b, n) in enumerate(zip(before, st.counts)):
            kv, there = plain.tokens(st.table, s, b + n)
            for got, want in zip((k, v), kv):
                want = np.where(there[b:, None, None], want[b:], 0)
                have = got[st.starts[s]:st.starts[s + 1]].cpu().numpy()
                assert np.array_equal(have, want.astype(np.float16))
        assert (k[-2:] == 7.5).all() and (v[-2:] == 7.5).all()


def test_a_captured_call_follows_lengths_and_positions(tt):
    D, H, heads = 128, 2, 8
    st = Step(213, D, H, 16, [30, 0], [40, 30], width=12)
    n = st.total
    x, pos, axis = torch.randn((n, heads + 2 * H, D), device="cuda"), torch.zeros((n, 3), dtype=torch.int32, device="cuda"), torch.arange(D // 2, device="cuda").remainder(3).byte()
    out, f = torch.empty((n, heads, D), dtype=torch.float16, device="cuda"), dev(INV[D])
    call = lambda o: tt.tetra_kv_append_at(x[:, :heads], x[:, heads:heads + H], x[:, heads + H:], *st.args(), pos, axis, o, f)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call(out)
    for lengths in ([30, 0], [47, 99], [0, 16]):
        st.d_lengths.copy_(i32(lengths))
        pos.random_(0, 5000)
        x.normal_()
        start = st.cache.clone()
        graph.replay()
        seen, made = out.clone(), st.cache.clone()
        st.cache.copy_(start)
        assert torch.equal(call(torch.empty_like(out)), seen) and torch.equal(st.cache, made)


def test_the_binding_refuses(tt):
    st = Step(214, 128, 2, 32, [40], [2])
    f, q, h = torch.zeros((2, 2, 128), device="cuda"), torch.zeros((2, 4, 128), device="cuda"), torch.zeros((2, 4, 128), dtype=torch.float16, device="cuda")
    pos, axis, inv = i32(np.zeros((2, 3))), torch.zeros(64, dtype=torch.uint8, device="cuda"), dev(INV[128])

    def refused(match, *args, **more):
        with pytest.raises(tt.TetraError, match=match):
            tt.tetra_kv_append_at(*args, **more)
    refused("positions: wrong", q, f, f, *st.args(), pos[:1], axis, h, inv)
    refused("positions: Long", q, f, f, *st.args(), pos.long(), axis, h, inv)
    refused("positions: wrong", q, f, f, *st.args(), pos[:, 0].contiguous(), axis, h, inv)
    refused("axis: wrong", q, f, f, *st.args(), pos, axis[:32], h, inv)
    refused("axis: Int", q, f, f, *st.args(), pos, axis.int(), h, inv)
    refused("axis: tensor is not on", q, f, f, *st.args(), pos, axis.cpu(), h, inv)
    refused("null", q, f, f, *st.args(), pos, axis, h, None)
    refused("out of range", q, f, f, *st.args(), i32(np.zeros((2, 9))), axis, h, inv)
    refused("null", q, f, f, *st.args(), i32(np.zeros((2, 0))), axis, h, inv)
    refused("inv_freq: Float", q, f, f, *st.args(), pos, axis, h, inv.float())
    refused("q and q_out", q, f, f, *st.args(), pos, axis, None, inv)
    refused("v: Half", q, f, f.half(), *st.args(), pos, axis, h, inv)
    none = torch.zeros((0, 4, 128), dtype=torch.float16, device="cuda")
    assert tt.tetra_kv_append_at(q[:0], f[:0], f[:0], *st.args(), pos[:0], axis, none, inv) is none


def test_as_many_rows_as_there_may_be(tt):
    """65536 rows of one sequence at once, read back: what tetra_kv_append makes of the same positions."""
    n, D = 65536, 64
    cache = tt.tetra_kv_cache(n // 64 + 1, 64, 1, D)
    table, starts, zero = torch.arange(n // 64 + 1, device="cuda", dtype=torch.int32).flip(0)[None], i32([0, n]), i32([7])
    x = torch.randn((n, 3, D), device="cuda")
    at = torch.arange(7, n + 7, device="cuda", dtype=torch.int32)[:, None].repeat(1, 2)
    axis = torch.arange(D // 2, device="cuda").remainder(2).byte()
    made = []
    for positions in (False, True):
        cache.fill_(0x81)
        q = torch.empty((n, 1, D), dtype=torch.float16, device="cuda")
        where = (cache, table, starts, zero)
        if positions:
            tt.tetra_kv_append_at(x[:, :1], x[:, 1:2], x[:, 2:], *where, at, axis, q, dev(INV[D]))
        else:
            tt.tetra_kv_append(x[:, :1], x[:, 1:2], x[:, 2:], *where, q, inv_freq=dev(INV[D]))
        k, v = (torch.empty((n, 1, D), dtype=torch.float16, device="cuda") for _ in range(2))
        tt.tetra_kv_read(*where, k, v)
        made.append((cache[..., :32 * D + 8].clone(), k, v, q))
    for a, b in list(zip(*made))[:3]:
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert (made[0][3].float() - made[1][3].float()).abs().max() <= 2.0 ** -10 * made[0][3].float().abs().max()
    step = made[0][0].view(-1, 32 * D + 8)[:, 32 * D:].contiguous().view(torch.float32).max()
    assert (made[1][2].float() - x[:, 2:]).abs().max() <= step * 0.5 + 2.0 ** -10 * x.abs().max()  # half a code, and float16's rounding
