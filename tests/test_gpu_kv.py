"""The paged cache and its attention on the GPU against the plain forms in 64 bits (step_reference.py): codes and scales are
equal, queries are rounded once, the attention stays within the bound that step_reference.attend derives."""
import numpy as np
import pytest
import torch

import step_reference as ref

pytestmark = pytest.mark.gpu

INV = {D: 1e6 ** (-np.arange(0, D, 2) / D) for D in (64, 128, 256)}


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return t.to("cuda", dtype) if dtype else t.cuda()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Step:
    """A cache full of earlier tokens and a step's sequences, on the device and as the plain form has them."""

    def __init__(self, seed, D, H, P, before, rows, width=None, spare=0, gap=0):
        self.rng = rng = np.random.default_rng(seed)
        self.D, self.H, self.P, self.spare = D, H, P, spare
        self.before, self.counts = list(before), list(rows)
        self.starts = np.concatenate([[0], np.cumsum(rows)])
        self.width = width or max(1, max(-(-max(1, b + n) // P) for b, n in zip(before, rows)))
        S = len(before)
        self.pages = S * self.width + 2
        self.table = rng.permutation(self.pages)[:S * self.width].reshape(S, self.width)
        codes = rng.integers(-127, 128, (2, self.pages, H, P // 16, 16, D)).astype(np.float64)
        scales = 2.0 ** rng.integers(-8, -2, (self.pages, H, P // 16, 2))
        self.raw = ref.pack(codes, scales, D)
        self.raw[..., 32 * D + 8:] = 0xA5  # bytes without meaning
        self.cache = dev(self.raw)
        self.gap = gap  # table rows lie apart
        t = np.full((S, self.width + gap), -7)
        t[:, :self.width] = self.table
        self.d_table = i32(t)[:, :self.width]
        self.d_starts, self.d_lengths = i32(self.starts), i32(self.before)

    @property
    def total(self):
        return int(self.starts[-1]) + self.spare

    def args(self):
        return self.cache, self.d_table, self.d_starts, self.d_lengths

    def plain(self):
        return ref.Cache(self.cache.cpu().numpy(), self.D, self.P)


def append_both(tt, st, heads, dtype=np.float32, norm=True, turn=True, spread=1.0, edit=None, sliced=True):
    """Appends random rows on the device and in the plain form; checks queries and the whole cache."""
    rng, n, D, H = st.rng, st.total, st.D, st.H
    x = (rng.standard_normal((n, heads + 2 * H, D)) * np.exp(spread * rng.standard_normal((n, heads + 2 * H, 1)))).astype(dtype)
    if edit:
        edit(x)
    q, k, v = x[:, :heads], x[:, heads:heads + H], x[:, heads + H:]
    w = [1 + 0.3 * rng.standard_normal(D).astype(np.float32) if norm else None for _ in range(2)]
    plain = st.plain()
    want = plain.append(q, k, v, st.table, st.starts, st.before, INV[D] if turn else None, w[0], w[1], 1e-6)
    d = dev(x)
    parts = [d[:, :heads], d[:, heads:heads + H], d[:, heads + H:]]
    if not sliced:
        parts = [p.contiguous() for p in parts]
    out = torch.full((n, heads, D), 7.5, dtype=torch.float16, device="cuda")
    got = tt.tetra_kv_append(*parts, *st.args(), out, inv_freq=dev(INV[D]) if turn else None, q_weight=dev(w[0]) if norm else None,
                             k_weight=dev(w[1]) if norm else None, eps=1e-6)
    assert got is out
    o = out.cpu().numpy().astype(np.float64)
    nobody = np.isnan(want).all((1, 2))
    nobody[:int(st.starts[-1])] = False
    assert (o[nobody] == 7.5).all()
    ok, have = want[~nobody], o[~nobody]
    fine = np.abs(ok) < 65520  # from there on float16 rounds to infinity
    # rounded once: half a step, relative 2^-11, or 2^-25 below the least normal number; 2^-40 for the 64-bit sums before
    assert (np.abs(have - ok)[fine] <= (2.0 ** -11 + 2.0 ** -40) * np.abs(ok[fine]) + 2.0 ** -25).all()
    assert not np.isfinite(have[~fine]).any()
    same_cache(st, plain)
    return plain


def same_cache(st, plain):
    raw = st.cache.cpu().numpy()
    codes, scales = ref.unpack(raw, st.D)
    assert np.array_equal(scales, plain.scales, equal_nan=True)
    live = live_tokens(st, codes.shape)
    bad = (codes != plain.codes) & live
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4])
    untouched = np.ones(raw.shape[:3], bool)
    for s, (b, n) in enumerate(zip(st.before, st.counts)):
        for pos in range(b, b + n):
            at = plain.place(st.table, s, pos)
            if at:
                untouched[at[0], :, at[1]] = False
    assert np.array_equal(raw[untouched], st.raw[untouched])
    assert (raw[..., 32 * st.D + 8:] == 0xA5).all()


def live_tokens(st, shape):
    """Tokens of the blocks that were written that are in the cache after the step, and all of the other blocks."""
    live = np.ones(shape, bool)
    plain = ref.Cache(st.raw, st.D, st.P)
    for s, (b, n) in enumerate(zip(st.before, st.counts)):
        if n and (at := plain.place(st.table, s, b + n - 1)):
            live[:, at[0], :, at[1], at[2] + 1:] = False
    return live


# ---- append -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,H,heads,P,before,rows", [
    (128, 8, 32, 64, [700], [1]),
    (128, 8, 40, 32, [0, 15, 16, 31, 32, 100], [1] * 6),
    (64, 2, 16, 16, [0, 3, 16, 47], [16, 14, 1, 2]),
    (256, 1, 7, 48, [5, 40], [50, 9]),           # a chunk over several blocks and a page
    (64, 1, 1, 16, [0], [1]),
    (128, 3, 3, 128, [127, 0, 255], [2, 0, 33]),  # a sequence without rows
    (128, 2, 24, 16, [11], [160]),
])
@pytest.mark.parametrize("dtype,norm,turn", [(np.float32, True, True), (np.float16, False, True), (np.float32, True, False), (np.float16, True, True)])
def test_append(tt, D, H, heads, P, before, rows, dtype, norm, turn):
    append_both(tt, Step(hash((D, H, heads, P)) % 1000, D, H, P, before, rows, spare=2, gap=3), heads, dtype, norm, turn)


def test_append_many_sequences(tt):
    rng = np.random.default_rng(3)
    n = 1024
    append_both(tt, Step(4, 64, 1, 16, rng.integers(0, 40, n).tolist(), rng.integers(0, 3, n).tolist()), 2, sliced=False)


def test_append_token_by_token_grows_scales(tt):
    """40 tokens of growing size, one a call: nearly every call grows a scale and rounds the block's codes again."""
    st = Step(5, 128, 2, 16, [0, 9], [1, 1], width=4)
    for i in range(40):
        st.raw = st.cache.cpu().numpy().copy()
        append_both(tt, st, 4, edit=lambda x: np.multiply(x, 1.3 ** i, out=x))
        st.before = [b + 1 for b in st.before]
        st.d_lengths = i32(st.before)


def test_append_takes_a_scale_that_is_not_a_power_of_two(tt):
    st = Step(6, 64, 2, 16, [5, 5, 5], [3, 2, 1])
    codes, scales = ref.unpack(st.raw, 64)
    scales = scales * np.float32(1.37)
    scales[st.table[1, 0]] = -1.0   # neither scale: counts as none
    scales[st.table[2, 0]] = 1e30   # larger than anything that comes
    st.raw[..., 32 * 64:32 * 64 + 8] = np.ascontiguousarray(scales).view(np.uint8)
    st.cache = dev(st.raw)
    append_both(tt, st, 2)


def test_append_zeros_and_tiny_and_huge(tt):
    def edit(x):
        x[0] = 0
        x[1] *= 2.0 ** -140 if x.dtype == np.float32 else 0
        x[2] = x[2] / np.abs(x[2]).max() * 3e38
        x[3] = 127 * 2.0 ** -20  # on the border of a scale
    st = Step(7, 128, 2, 32, [0, 16, 32, 0, 3], [1] * 5)
    append_both(tt, st, 4, norm=False, turn=False, edit=edit)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_append_of_what_is_not_finite_spoils_its_block_alone(tt, bad):
    st = Step(8, 64, 2, 16, [5, 20, 16], [2, 1, 17])

    def edit(x):
        x[0, 2, 7] = bad       # a key of head 0 (behind two query heads)
        x[2, 5, 3] = bad       # a value of head 1
        x[3, 3, 1] = bad       # a key of head 1 in the first of a chunk's two blocks
    append_both(tt, st, 2, norm=False, turn=False, edit=edit)
    # ... from then on, until the block is begun anew
    st.raw, st.before, st.counts = st.cache.cpu().numpy().copy(), [7, 21, 32], [1, 1, 1]
    st.starts = np.array([0, 1, 2, 3])
    st.d_starts, st.d_lengths = i32(st.starts), i32(st.before)
    plain = append_both(tt, st, 2)
    assert np.isnan(plain.scales).any()
    st.raw, st.before, st.counts = st.cache.cpu().numpy().copy(), [0, 16, 16], [1, 1, 1]
    st.d_lengths = i32(st.before)
    plain = append_both(tt, st, 2)
    assert not np.isnan(plain.scales).any()


def test_append_places_that_are_not_there(tt):
    """No slot, positions behind the table, page numbers out of range: the queries come, nothing is stored."""
    st = Step(9, 128, 2, 16, [-3, 30, 2 ** 31 - 3, 40, 17, -2 ** 31], [2, 5, 1, 1, 1, 1], width=2)
    st.table[3] = [-1, -2 ** 31]
    st.table[4] = [0, st.pages]
    st.d_table = i32(st.table)
    append_both(tt, st, 4)
    st = Step(10, 64, 1, 32, [-5], [20], width=1)  # from before the first position into the first block
    append_both(tt, st, 1)


def test_ranges_of_rows_that_make_no_sense_have_no_rows(tt):
    st = Step(11, 64, 2, 16, [3, 3, 3], [1, 1, 1])
    h = torch.ones((3, 2, 64), device="cuda")
    before = st.cache.clone()
    out = torch.full((3, 2, 64), 7.5, dtype=torch.float16, device="cuda")
    for starts in ([-1, -1, -1, -1], [2, 1, 0, -5], [4, 5, 6, 7], [0, 9, 9, 9], [-2 ** 31, 2 ** 31 - 1, -1, 0]):
        st.d_starts = i32(starts)
        tt.tetra_kv_append(h, h, h, *st.args(), out)
        tt.tetra_kv_read(*st.args(), out, out)
        tt.tetra_kv_attend(out, *st.args(), out, tt.tetra_kv_workspace(64))
        assert torch.equal(st.cache, before) and (out == 7.5).all(), starts


def test_append_without_queries(tt):
    st, other = (Step(12, 128, 2, 32, [9, 60], [3, 1]) for _ in range(2))
    x = torch.randn((4, 2, 2, 128), device="cuda")
    assert tt.tetra_kv_append(None, x[:, 0], x[:, 1], *st.args(), None, inv_freq=dev(INV[128])) is None
    q = torch.randn((4, 6, 128), device="cuda")
    tt.tetra_kv_append(q, x[:, 0], x[:, 1], *other.args(), torch.empty((4, 6, 128), dtype=torch.float16, device="cuda"), inv_freq=dev(INV[128]))
    assert torch.equal(st.cache, other.cache)


def test_far_positions_keep_their_angle(tt):
    """Two million tokens on, with a table that has one page for all of it."""
    st = Step(13, 128, 1, 16, [2000003], [2], width=1)
    st.table = np.full((1, 2000016 // 16), st.table[0, 0])
    st.width, st.d_table = st.table.shape[1], i32(st.table)
    append_both(tt, st, 2)


# ---- read -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,H,P", [(64, 2, 16), (128, 8, 48), (256, 3, 32)])
def test_read(tt, D, H, P):
    st = Step(14, D, H, P, [0, 5, 16, 30, -3], [40, 12, 1, 3, 5], width=40 // P + 1, spare=2)
    st.table[3] = -1
    st.d_table = i32(st.table)
    k, v = (torch.full((st.total, H, D), 7.5, dtype=torch.float16, device="cuda") for _ in range(2))
    got = tt.tetra_kv_read(*st.args(), k, v)
    assert got[0] is k and got[1] is v
    plain = st.plain()
    for s, (a, b) in enumerate(zip(st.starts, st.starts[1:])):
        kv, _ = plain.tokens(st.table, s, st.before[s] + b - a)
        lo = max(0, st.before[s])
        for which, t in ((0, k), (1, v)):
            have = t[a:b].cpu().numpy()
            want = np.zeros(have.shape)
            want[lo - st.before[s]:] = kv[which, lo:]
            assert np.array_equal(have, want.astype(np.float16)), s  # code * scale: seven bits, exact
    assert (k[st.starts[-1]:] == 7.5).all() and (v[st.starts[-1]:] == 7.5).all()


# ---- attend -----------------------------------------------------------------------------------------------------------
def attend_check(tt, st, heads, scale=None, q=None, workspace=None, plain=None):
    n, D = st.total, st.D
    if q is None:
        q = st.rng.standard_normal((n, heads, D)).astype(np.float16)
    out = torch.full((n, heads, D), 7.5, dtype=torch.float16, device="cuda")
    ws = workspace if workspace is not None else tt.tetra_kv_workspace(D)
    d = dev(q)
    assert tt.tetra_kv_attend(d, *st.args(), out, ws, scale) is out
    want, bound = ref.attend(plain or st.plain(), q, st.table, st.starts, st.before, 1 / np.sqrt(D) if scale is None else scale)
    have = out.cpu().numpy().astype(np.float64)
    nobody = np.isnan(bound).all((1, 2)) & (np.arange(n) >= st.starts[-1])
    assert (have[nobody] == 7.5).all()
    have, want, bound = have[~nobody], want[~nobody], bound[~nobody]
    finite = np.isfinite(want)
    assert np.array_equal(np.isfinite(have), finite)
    worst = np.abs(have - want)[finite] / np.maximum(bound[finite], 1e-300)
    worst[np.abs(have - want)[finite] == 0] = 0
    assert worst.size == 0 or worst.max() <= 1, worst.max()
    assert not ws[:4608].any()  # the counters are zero again
    again = torch.full_like(out, 7.5)
    tt.tetra_kv_attend(d, *st.args(), again, ws, scale)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    return out


@pytest.mark.parametrize("D,H,heads,P", [(128, 8, 32, 64), (128, 8, 40, 32), (64, 2, 16, 16), (256, 1, 7, 48), (128, 2, 2, 128), (256, 2, 24, 16), (64, 1, 9, 32), (128, 1, 20, 16)])
@pytest.mark.parametrize("before,rows", [([0], [1]), ([1], [1]), ([14, 15, 16, 17], [1] * 4), ([256], [1]), ([0, 700, 3, 1500, 127], [1] * 5)])
def test_attend_single_tokens(tt, D, H, heads, P, before, rows):
    attend_check(tt, Step(20, D, H, P, before, rows, spare=1, gap=1), heads)


@pytest.mark.parametrize("D,H,heads,P", [(128, 8, 32, 64), (128, 2, 10, 16), (64, 2, 16, 16), (256, 1, 7, 48), (64, 4, 4, 32)])
@pytest.mark.parametrize("before,rows", [([0], [16]), ([5, 0, 300], [16, 7, 2]), ([15], [2]), ([100, 40], [1, 37]), ([0], [130]), ([33, 33, 33], [0, 5, 0])])
def test_attend_chunks_are_causal(tt, D, H, heads, P, before, rows):
    attend_check(tt, Step(21, D, H, P, before, rows, spare=1), heads)


def test_attend_long(tt):
    """Many CTAs to an item, and items that begin and end inside ranges."""
    attend_check(tt, Step(22, 128, 2, 64, [30011], [1]), 8)
    attend_check(tt, Step(23, 128, 1, 16, [20000, 3, 9000], [4, 1, 16]), 5)
    attend_check(tt, Step(24, 64, 8, 128, [5001, 4097, 1, 2900], [1] * 4), 16)
    attend_check(tt, Step(25, 256, 1, 64, [9000], [3]), 4)


def test_attend_many_sequences(tt):
    rng = np.random.default_rng(26)
    attend_check(tt, Step(26, 64, 2, 16, rng.integers(-2, 60, 1024).tolist(), rng.integers(0, 3, 1024).tolist()), 4)
    attend_check(tt, Step(27, 128, 8, 16, rng.integers(0, 100, 300).tolist(), [1] * 300), 32)


@pytest.mark.parametrize("seqs,H,long,short", [(95, 2, 640, 640), (74, 2, 600, 1100), (100, 1, 513, 1100), (37, 8, 520, 500), (148, 2, 300, 1030), (50, 5, 40, 40), (33, 4, 3000, 10), (20, 7, 600, 1200), (32, 9, 640, 640),
                                                   (400, 3, 40, 17), (64, 8, 3, 3), (30, 16, 100, 1), (64, 8, 130, 200), (700, 7, 20, 33)])
def test_attend_at_every_way_to_cut(tt, seqs, H, long, short):
    """Items about as many as CTAs, parts that just fit or just do not, equal and ragged ones."""
    attend_check(tt, Step(37 + seqs, 64, H, 64, [long - 3 * i % 17 if i % 2 else short for i in range(seqs)], [1] * seqs), 2 * H)


@pytest.mark.parametrize("D,H,heads,seqs,rows", [(64, 8, 64, 700, 4), (256, 4, 48, 200, 3), (128, 6, 60, 300, 2)])
def test_attend_many_chunks(tt, D, H, heads, seqs, rows):
    """More parts of items to a CTA than it looks up at a time."""
    attend_check(tt, Step(38 + D, D, H, 16, [i * 7 % 23 for i in range(seqs)], [rows - (i % 11 == 0) for i in range(seqs)], spare=2), heads)


def test_a_long_prompt_in_one_call(tt):
    """Far more rows of a sequence than a product takes: slow, and right."""
    attend_check(tt, Step(39, 64, 2, 64, [100, 3], [700, 1]), 6)


def test_attend_in_place(tt):
    """The output may lie where the queries were: a column is read before it is written."""
    st = Step(43, 128, 2, 32, [3000, 5, 400], [1, 2, 16])
    q = st.rng.standard_normal((19, 8, 128)).astype(np.float16)
    ws, d = tt.tetra_kv_workspace(128), dev(q)
    want = tt.tetra_kv_attend(d, *st.args(), torch.empty_like(d), ws)
    assert torch.equal(tt.tetra_kv_attend(d, *st.args(), d, ws), want)


def test_attend_rows_that_see_nothing(tt):
    st = Step(28, 128, 2, 16, [-1, -5, 20, 7, -2], [1, 3, 1, 1, 5], width=2)
    st.table[2] = [-1, 10 ** 6]
    st.d_table = i32(st.table)
    out = attend_check(tt, st, 8)
    assert not out[:5].any() and not out[6:8].any() and out[8].any()


def test_attend_leaves_out_pages_that_are_not_there(tt):
    st = Step(29, 128, 2, 32, [500, 90], [2, 16])
    st.table[0, 3] = -1
    st.table[0, 15] = st.pages  # the page of the newest tokens too
    st.table[1, 0] = 2 ** 31 - 1
    st.d_table = i32(st.table)
    attend_check(tt, st, 8)


def test_attend_behind_the_table(tt):
    """Lengths beyond what the table holds: the tokens that have a place are seen."""
    attend_check(tt, Step(30, 64, 1, 16, [100, 2 ** 31 - 2], [3, 1], width=3), 4)


def test_nothing_that_is_not_seen_is_felt(tt):
    """NaN scales in every page that no sequence has, in blocks behind the last token, in the newest block for the rows before it; any bytes behind the last token."""
    st = Step(31, 128, 2, 32, [40, 14], [1, 3])
    codes, scales = ref.unpack(st.raw, 128)
    used = np.zeros(st.raw.shape[:3], bool)
    for s, n in ((0, 41), (1, 17)):
        for pos in range(0, n, 16):
            used[st.table[s, pos // 32], :, pos % 32 // 16] = True
    scales[~used] = np.nan
    scales[st.table[1, 0], :, 1] = np.nan  # position 16, the third row's own
    st.raw = ref.pack(codes, scales, 128)
    for s, n in ((0, 41), (1, 17)):  # codes behind the last token: any byte, 0 among them
        at = ref.byte_places(128)
        for place in at:
            st.raw[st.table[s, n // 32], :, n % 32 // 16][:, place[n % 16:].reshape(-1)] = 0
    st.cache = dev(st.raw)
    out = attend_check(tt, st, 8).cpu().numpy()
    assert np.isfinite(out[:3]).all() and np.isnan(out[3]).all()


def test_a_query_that_is_not_finite_stays_alone(tt):
    st = Step(32, 128, 2, 32, [40, 14], [2, 1])
    q = st.rng.standard_normal((3, 8, 128)).astype(np.float16)
    q[1, 2, 5] = np.nan
    attend_check(tt, st, 8, q=q)


@pytest.mark.parametrize("case", ["values", "keys", "zeros", "rising", "far"])
def test_scales_of_very_different_size(tt, case):
    st = Step(33, 128, 2, 16, [200, 77], [1, 4])
    codes, scales = ref.unpack(st.raw, 128)
    n = np.arange(scales[..., 0].size).reshape(scales.shape[:3])
    if case == "values":       # large values where the weights are small
        scales[..., 1] = 2.0 ** (n % 5 * 4 - 16)
    elif case == "keys":       # scores from flat to one token that takes all
        scales[..., 0] = 2.0 ** (n % 7 - 7)
    elif case == "zeros":      # blocks of zeros, keys or values
        scales[..., 1] *= n % 3 > 0
        scales[..., 0] *= n % 4 > 0
    elif case == "rising":     # every block moves the reference
        for s in range(2):
            scales[st.table[s], :, 0, 1] = 2.0 ** (np.arange(st.width) * 2 - 20)[:, None]
    else:                      # below what float16 shows, but for some
        scales[..., 1] = np.where(n % 4 == 0, 2.0 ** -9, 2.0 ** -90)
    st.raw = ref.pack(codes, scales, 128)
    st.cache = dev(st.raw)
    attend_check(tt, st, 8, scale=0.02)


def test_all_values_zero_and_scale_zero_or_negative(tt):
    st = Step(34, 64, 2, 16, [50], [2])
    codes, scales = ref.unpack(st.raw, 64)
    attend_check(tt, st, 4, scale=0.0)
    attend_check(tt, st, 4, scale=-0.05)
    scales[..., 1] = 0
    st.raw = ref.pack(codes, scales, 64)
    st.cache = dev(st.raw)
    assert not attend_check(tt, st, 4).any()


def test_rows_of_queries_may_lie_apart(tt):
    st = Step(35, 128, 2, 32, [40, 14], [2, 1])
    big = torch.randn((3, 12, 128), device="cuda").half()
    out, want = (torch.empty((3, 8, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    ws = tt.tetra_kv_workspace(128)
    tt.tetra_kv_attend(big[:, 2:10], *st.args(), out, ws)
    tt.tetra_kv_attend(big[:, 2:10].contiguous(), *st.args(), want, ws)
    assert torch.equal(out, want)


def test_offsets_that_pass_32_bits(tt):
    """A cache of 4.6 GB; the sequences live at its end, and one page of them at its beginning."""
    D, H, P = 128, 8, 128
    pages = 17600
    st = Step(36, D, H, P, [300, 130], [1, 2])
    cache = torch.empty((pages, H, P // 16, 32 * D + 16), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32
    moved = pages - 1 - st.table
    moved[0, 0] = 0
    raw = torch.from_numpy(st.raw).cuda()
    for old, new in zip(st.table.reshape(-1), moved.reshape(-1)):
        cache[new] = raw[old]
    small = st.plain()
    q = st.rng.standard_normal((3, 32, D)).astype(np.float32)
    kv = st.rng.standard_normal((2, 3, H, D)).astype(np.float32)
    want = small.append(q, kv[0], kv[1], st.table, st.starts, st.before, INV[D])
    out = torch.empty((3, 32, D), dtype=torch.float16, device="cuda")
    big = (cache, i32(moved), st.d_starts, st.d_lengths)
    tt.tetra_kv_append(dev(q), dev(kv[0]), dev(kv[1]), *big, out, inv_freq=dev(INV[D]))
    have = out.cpu().numpy()
    assert (np.abs(have - want) <= (2.0 ** -11 + 2.0 ** -40) * np.abs(want) + 2.0 ** -25).all()
    for old, new in zip(st.table.reshape(-1), moved.reshape(-1)):
        st.cache[old] = cache[new]
    same_cache(st, small)
    a = tt.tetra_kv_attend(out, *big, torch.empty_like(out), tt.tetra_kv_workspace(D))
    o, bound = ref.attend(small, have, st.table, st.starts, st.before, 1 / np.sqrt(D))
    assert (np.abs(a.cpu().numpy() - o) <= bound).all()


# ---- streams, graphs, refusals -----------------------------------------------------------------------------------------
def test_a_captured_step_follows_lengths_and_pages(tt):
    """append and attend in one graph, replayed while a sequence grows by what the graph appends, beside eager calls."""
    D, H, heads = 128, 2, 8
    st = Step(40, D, H, 16, [30, 0], [1, 1], width=4)
    x = torch.randn((2, heads + 2 * H, D), device="cuda")
    q, out, ws = torch.empty((2, heads, D), dtype=torch.float16, device="cuda"), torch.empty((2, heads, D), dtype=torch.float16, device="cuda"), tt.tetra_kv_workspace(D)
    f = dev(INV[D])

    def step():
        tt.tetra_kv_append(x[:, :heads], x[:, heads:heads + H], x[:, heads + H:], *st.args(), q, inv_freq=f)
        tt.tetra_kv_attend(q, *st.args(), out, ws)
        st.d_lengths += 1
    side = torch.cuda.Stream()
    start, lengths = st.cache.clone(), st.d_lengths.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    assert torch.equal(start, st.cache)
    seen = []
    rows = [torch.randn_like(x) for _ in range(20)]
    for r in rows:
        x.copy_(r)
        graph.replay()
        seen.append(out.clone())
    torch.cuda.synchronize()
    st.cache.copy_(start)
    st.d_lengths.copy_(lengths)
    for r, want in zip(rows, seen):
        x.copy_(r)
        step()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))


def test_two_streams_with_workspaces_of_their_own(tt):
    st = Step(41, 128, 2, 64, [9000], [1])
    q = torch.randn((1, 8, 128), device="cuda").half()
    want = tt.tetra_kv_attend(q, *st.args(), torch.empty_like(q), tt.tetra_kv_workspace(128))
    streams, ws, outs = [torch.cuda.Stream() for _ in range(2)], [tt.tetra_kv_workspace(128) for _ in range(2)], [[torch.empty_like(q) for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                tt.tetra_kv_attend(q, *st.args(), outs[k][i], ws[k])
    torch.cuda.synchronize()
    for o in outs[0] + outs[1]:
        assert torch.equal(o, want)
    other = torch.empty_like(q)
    tt.tetra_kv_attend(q, *st.args(), other, ws[0], stream=streams[1])
    streams[1].synchronize()
    assert torch.equal(other, want)


def test_the_binding_refuses(tt):
    st = Step(42, 128, 2, 32, [40], [2])
    cache, table, starts, lengths = st.args()
    f = torch.zeros((2, 2, 128), device="cuda")
    q, h, ws = torch.zeros((2, 4, 128), device="cuda"), torch.zeros((2, 4, 128), dtype=torch.float16, device="cuda"), tt.tetra_kv_workspace(128)
    a = tt.tetra_kv_append

    def refused(match, call, *args, **more):
        with pytest.raises(tt.TetraError, match=match):
            call(*args, **more)
    refused("v: Half", a, q, f, f.half(), cache, table, starts, lengths, h)
    refused("q: Half", a, q.half(), f, f, cache, table, starts, lengths, h)
    refused("k: wrong shape", a, q, f[:, :1], f, cache, table, starts, lengths, h)
    refused("v: wrong shape", a, q, f, f[:1], cache, table, starts, lengths, h)
    refused("k: the heads", a, q, f.transpose(1, 2).contiguous().transpose(1, 2), f, cache, table, starts, lengths, h)
    refused("v: rows overlap", a, q, f, f[:1].expand(2, 2, 128), cache, table, starts, lengths, h)
    refused("q and q_out", a, q, f, f, cache, table, starts, lengths, None)
    refused("q_out: wrong shape", a, q, f, f, cache, table, starts, lengths, h[:1])
    refused("q_out: Float", a, q, f, f, cache, table, starts, lengths, q)
    refused("out of range", a, torch.zeros((2, 3, 128), device="cuda"), f, f, cache, table, starts, lengths, h[:, :3].contiguous())
    refused("inv_freq: Float", a, q, f, f, cache, table, starts, lengths, h, inv_freq=torch.zeros(64, device="cuda"))
    refused("inv_freq: wrong", a, q, f, f, cache, table, starts, lengths, h, inv_freq=torch.zeros(128, dtype=torch.float64, device="cuda"))
    refused("k_weight: wrong", a, q, f, f, cache, table, starts, lengths, h, k_weight=torch.zeros(64, device="cuda"))
    refused("out of range", a, q, f, f, cache, table, starts, lengths, h, eps=-1.0)
    refused("cache: wrong shape", a, q, f, f, cache[:, :, :, :-16], table, starts, lengths, h)
    refused("page_table: Long", a, q, f, f, cache, table.long(), starts, lengths, h)
    refused("row_start: wrong", a, q, f, f, cache, table, starts[:1], lengths, h)
    refused("lengths: wrong", a, q, f, f, cache, table, starts, starts, h)
    refused("k: wrong shape", a, q, f[:, :, :64], f, cache, table, starts, lengths, h)
    refused("k_out: wrong", tt.tetra_kv_read, cache, table, starts, lengths, h, h)
    refused("v_out: Float", tt.tetra_kv_read, cache, table, starts, lengths, f.half(), f)
    b = tt.tetra_kv_attend
    refused("q: Float", b, q, cache, table, starts, lengths, h, ws)
    refused("out: wrong", b, h, cache, table, starts, lengths, h[:1], ws)
    refused("buffer too small", b, h, cache, table, starts, lengths, h, ws[:-1])
    refused("workspace: Float", b, h, cache, table, starts, lengths, h, ws.float())
    refused("out of range", b, h, cache, table, starts, lengths, h, ws, float("nan"))
    refused("misaligned", b, torch.zeros((2, 4 * 128 + 4), dtype=torch.float16, device="cuda")[:, 4:].view(2, 4, 128), cache, table, starts, lengths, h, ws)
    refused("misaligned", b, h, cache, table, starts, lengths, h, torch.zeros(ws.numel() + 16, dtype=torch.uint8, device="cuda")[16:])
    many = torch.zeros((1025, 1), dtype=torch.int32, device="cuda")
    refused("out of range", b, h, cache, many, torch.zeros(1026, dtype=torch.int32, device="cuda"), many[:, 0].contiguous(), h, ws)
    # no rows: nothing to do
    none = torch.zeros((0, 4, 128), dtype=torch.float16, device="cuda")
    assert b(none, cache, table, starts, lengths, none, ws) is none
    assert a(q[:0], f[:0], f[:0], cache, table, starts, lengths, none) is none
