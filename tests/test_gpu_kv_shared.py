"""Attention of sequences that begin with the same tokens, against the plain form in 64 bits, which knows nothing of groups.

The bound is step_reference.attend's, for these differences.  A reference is a whole number, so the largest weight times scale lies
between 2^6.5 and 2^15, not 2^7: a weight of less than float16's least normal number is off by 2^-31.5 of the largest, not 2^-32, which is
less than twice that term.  Sums of n tokens are added up 16 tokens at a time and then piece by piece, in float32 by the tensor
cores, which may cut where they round: (n / 16 + 64) 2^-23 of the mean of |v|, of which the bound holds 2^-11 times: the bound times
(n / 16 + 64) 2^-12."""
import numpy as np
import pytest
import torch

import step_reference as ref
from test_gpu_kv import Step, dev, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def wide(st, table):
    """A table with room for more tokens and sequences than there are, the others without rows: what a call could save is judged by that."""
    n = len(table)
    idle = max(0, 24 - n) if st.total <= 2 * n else 0
    room = int(126e6 + 160 * st.total * 64 * st.D) // (st.H * max(900, (n + idle) * st.D) * st.P) + 1
    st.d_starts, st.d_lengths = i32(list(st.starts) + [st.starts[-1]] * idle), i32(list(st.before) + [0] * idle)
    t = np.concatenate([table, np.full((n, max(st.gap, room)), -7)], 1)
    return i32(np.concatenate([t, np.full((idle, t.shape[1]), -7)]))[:, :max(st.width, room)]


def share(st, groups, narrow=False):
    """groups: (first sequence, the one behind the last, tokens): their table entries become the first one's."""
    for a, b, n in groups:
        pages = min(max(n, 0) // st.P, st.width)
        if b > a:
            st.table[a:b, :pages] = st.table[a, :pages]
    st.d_table = i32(np.concatenate([st.table, np.full((len(st.table), st.gap), -7)], 1))[:, :st.width] if narrow else wide(st, st.table)
    start = [g[0] for g in groups] + [groups[-1][1] if groups else 0]
    return i32(start), i32([g[2] for g in groups])


def shared_check(tt, st, heads, groups, scale=None, q=None, workspace=None, plain=None, narrow=False):
    n, D = st.total, st.D
    start, shared = share(st, groups, narrow)
    if q is None:
        q = st.rng.standard_normal((n, heads, D)).astype(np.float16)
    out = torch.full((n, heads, D), 7.5, dtype=torch.float16, device="cuda")
    ws = workspace if workspace is not None else tt.tetra_kv_shared_workspace(D, n, heads, st.H, len(groups))
    d = dev(q)
    assert tt.tetra_kv_attend_shared(d, *st.args(), start, shared, out, ws, scale) is out
    want, bound = ref.attend(plain or st.plain(), q, st.table, st.starts, st.before, 1 / np.sqrt(D) if scale is None else scale)
    longest = max([b + c for b, c in zip(st.before, st.counts)] + [0])
    bound = bound * (2 + (longest / 16 + 64) * 2.0 ** -12)
    have = out.cpu().numpy().astype(np.float64)
    nobody = np.isnan(bound).all((1, 2)) & (np.arange(n) >= st.starts[-1])
    assert (have[nobody] == 7.5).all()
    have, want, bound = have[~nobody], want[~nobody], bound[~nobody]
    finite = np.isfinite(want)
    assert not np.isfinite(have[~finite]).any()
    over = ~np.isfinite(have)  # what float16 does not hold
    assert not np.isnan(have[finite]).any() and (np.abs(want) + bound >= 65504)[over & finite].all()
    finite &= ~over
    worst = np.abs(have - want)[finite] / np.maximum(bound[finite], 1e-300)
    worst[np.abs(have - want)[finite] == 0] = 0
    assert worst.size == 0 or worst.max() <= 1, worst.max()
    again = torch.full_like(out, 7.5)
    tt.tetra_kv_attend_shared(d, *st.args(), start, shared, again, ws, scale)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    return out


# Heads of every size and group; tokens from one step of the products to many, ends inside a step, a block and a page.
@pytest.mark.parametrize("D,H,heads,P", [(128, 8, 32, 64), (128, 8, 40, 32), (64, 2, 16, 16), (256, 1, 7, 48), (128, 2, 2, 128), (256, 2, 24, 16), (64, 1, 9, 32), (128, 1, 20, 16)])
@pytest.mark.parametrize("shared,before", [(128, [128, 128]), (144, [150, 144, 1000]), (200, [192, 300]), (1000, [1000, 1003, 1100, 1001]), (2047, [2047, 2100])])
def test_single_tokens(tt, D, H, heads, P, shared, before):
    shared -= shared % P  # whole pages are the same
    shared_check(tt, Step(101, D, H, P, [max(b, shared) for b in before], [1] * len(before)), heads, [(0, len(before), shared)])


# Columns of a head: below, at and above what a slot, a tile and two tiles have.
@pytest.mark.parametrize("seqs,heads,H,D", [(31, 8, 2, 128), (32, 8, 2, 128), (33, 8, 2, 128), (64, 4, 1, 128), (65, 4, 1, 128), (200, 2, 1, 64), (127, 1, 1, 64), (129, 1, 1, 64), (40, 4, 1, 256), (26, 10, 2, 256)])
def test_columns(tt, seqs, heads, H, D):
    rng = np.random.default_rng(seqs)
    shared_check(tt, Step(102, D, H, 16, (320 + rng.integers(0, 60, seqs)).tolist(), [1] * seqs), heads, [(0, seqs, 320)])


@pytest.mark.parametrize("D,H,heads,P", [(128, 8, 32, 64), (64, 2, 16, 16), (256, 1, 7, 48)])
@pytest.mark.parametrize("shared,before,rows", [(192, [192, 192, 200], [5, 1, 16]), (480, [480, 500], [37, 3]), (144, [144, 144, 144, 144], [0, 12, 0, 9])])
def test_chunks_are_causal(tt, D, H, heads, P, shared, before, rows):
    shared -= shared % P
    shared_check(tt, Step(103, D, H, P, before, rows, spare=2, gap=3), heads, [(0, len(before), shared)])


def test_several_groups_and_sequences_in_none(tt):
    before = [40, 700, 300, 310, 290, 17, 500, 520, 501, 999]
    st = Step(104, 128, 2, 16, before, [1] * len(before), spare=3)
    shared_check(tt, st, 8, [(2, 5, 288), (5, 5, 100), (5, 6, 16), (6, 9, 496)])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_many_groups(tt, D):
    """More groups than a warp has lanes, more items than the grid has CTAs."""
    rng = np.random.default_rng(105)
    groups, before = [], []
    for _ in range(90):
        n, tokens = int(rng.integers(1, 4)), int(rng.integers(0, 12)) * 32
        groups.append((len(before), len(before) + n, tokens))
        before += [tokens + int(rng.integers(0, 40)) for _ in range(n)]
    shared_check(tt, Step(105, D, 4, 32, before, [1] * len(before)), 8, groups)


@pytest.mark.parametrize("D,H,heads,P", [(128, 8, 32, 64), (64, 2, 16, 16), (256, 1, 7, 48)])
@pytest.mark.parametrize("shared,before,rows", [(192, [192, 192, 200], [5, 1, 16]), (960, [960, 1000], [1, 1])])
def test_tables_without_room_for_more(tt, D, H, heads, P, shared, before, rows):
    """Too little to save: one launch, and the bits of tetra_kv_attend."""
    st = Step(113, D, H, P, before, rows)
    q = st.rng.standard_normal((st.total, heads, D)).astype(np.float16)
    out = shared_check(tt, st, heads, [(0, len(before), shared)], q=q, narrow=True)
    assert torch.equal(out, tt.tetra_kv_attend(dev(q), *st.args(), torch.empty_like(out), tt.tetra_kv_workspace(D)))


def test_as_many_sequences_as_there_may_be(tt):
    n = 1024
    st = Step(106, 64, 1, 16, [160] * n, [1] * n)
    shared_check(tt, st, 2, [(0, 500, 160), (500, 1024, 144)])


def test_a_group_for_each_sequence_and_none_at_all(tt):
    st = Step(107, 128, 2, 16, [200, 200, 33], [1] * 3)
    shared_check(tt, st, 8, [(i, i + 1, 192) for i in range(3)])
    q = st.rng.standard_normal((3, 8, 128)).astype(np.float16)
    ws = tt.tetra_kv_shared_workspace(128, 3, 8, 2, 0)
    none = tt.tetra_kv_attend_shared(dev(q), *st.args(), i32([0]), i32([]), torch.empty((3, 8, 128), dtype=torch.float16, device="cuda"), ws)
    alone = tt.tetra_kv_attend(dev(q), *st.args(), torch.empty_like(none), tt.tetra_kv_workspace(128))
    assert torch.equal(none, alone)


def test_sequences_that_do_not_take_part(tt):
    """Shorter than what is shared, without rows, without a sequence: the others share nevertheless."""
    before = [400, 100, 399, -1, 450, 0, -7, 512]
    st = Step(108, 128, 2, 16, before, [1, 1, 2, 1, 0, 3, 9, 1])
    shared_check(tt, st, 8, [(0, 8, 400)])
    shared_check(tt, st, 8, [(0, 8, 100000)])
    shared_check(tt, st, 8, [(0, 8, -5)])
    shared_check(tt, Step(109, 128, 2, 16, [-1, -1, -1], [1, 1, 1]), 8, [(0, 3, 160)])


def test_groups_that_make_no_sense_share_nothing(tt):
    st = Step(110, 64, 2, 16, [300, 300, 300], [1] * 3)
    st.table[:, :16] = st.table[0, :16]
    st.d_table = wide(st, st.table)
    q = dev(st.rng.standard_normal((3, 4, 64)).astype(np.float16))
    want, bound = ref.attend(st.plain(), q.cpu().numpy(), st.table, st.starts, st.before, 1 / 8)
    for start in ([-2, 3], [0, 4], [2, 1], [3, 3], [0, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1], [1, 0, 3], [0, 5, 2]):
        ws = tt.tetra_kv_shared_workspace(64, 3, 4, 2, len(start) - 1)
        out = tt.tetra_kv_attend_shared(q, *st.args(), i32(start), i32([256] * (len(start) - 1)), torch.empty((3, 4, 64), dtype=torch.float16, device="cuda"), ws)
        assert (np.abs(out.cpu().numpy() - want) <= 3 * bound).all(), start


def test_ranges_of_rows_that_make_no_sense_have_no_rows(tt):
    st = Step(111, 64, 2, 16, [200] * 4, [1] * 4)
    start, shared = share(st, [(0, 4, 192)])
    q = torch.randn((4, 4, 64), device="cuda").half()
    ws = tt.tetra_kv_shared_workspace(64, 4, 4, 2, 1)
    for starts, live in (([0, 1, 1, 2, 9], [0, 1]), ([-1, 1, 2, 3, 4], [1, 2, 3]), ([4, 4, 4, 4, 4], []), ([9, 9, 9, 9, 9], [])):
        out = torch.full_like(q, 7.5)
        tt.tetra_kv_attend_shared(q, st.cache, st.d_table, i32(starts + starts[-1:] * (len(st.d_lengths) - 4)), st.d_lengths, start, shared, out, ws)
        rows = torch.zeros(4, dtype=torch.bool, device="cuda")
        rows[live] = True
        assert (out[~rows] == 7.5).all() and (out[rows] != 7.5).any(-1).all(), starts


def test_pages_that_are_not_there(tt):
    st = Step(112, 128, 2, 16, [330, 340, 333], [1] * 3)
    share(st, [(0, 3, 320)])
    st.table[:, 3], st.table[:, 7], st.table[1, 20] = -1, st.pages, 2 ** 31 - 1
    shared_check(tt, st, 8, [(0, 3, 320)])
    st.table[:, :20] = -3  # nothing of what is shared
    shared_check(tt, st, 8, [(0, 3, 320)])
    st.table[:] = -3
    assert not shared_check(tt, st, 8, [(0, 3, 320)]).any()


@pytest.mark.parametrize("case", ["values", "keys", "zeros", "rising", "falling", "far"])
@pytest.mark.parametrize("D,seqs", [(128, 3), (128, 40), (64, 5), (256, 4)])
def test_scales_of_very_different_size(tt, case, D, seqs):
    st = Step(113, D, 1, 16, [400] * seqs, [1] * seqs)
    share(st, [(0, seqs, 384)])
    codes, scales = ref.unpack(st.raw, D)
    n = np.arange(scales[..., 0].size).reshape(scales.shape[:3])
    if case == "values":       # large values where the weights are small
        scales[..., 1] = 2.0 ** (n % 5 * 4 - 16)
    elif case == "keys":       # scores from flat to one token that takes all
        scales[..., 0] = 2.0 ** (n % 7 - 7)
    elif case == "zeros":      # blocks of zeros, keys or values
        scales[..., 1] *= n % 3 > 0
        scales[..., 0] *= n % 4 > 0
    elif case in ("rising", "falling"):  # every block moves the reference, or none but the first
        steps = np.arange(24) if case == "rising" else np.arange(24)[::-1]
        scales[st.table[0, :24], :, 0, 1] = 2.0 ** (steps * 2 - 20)[:, None]
    else:                      # below what float16 shows, but for some
        scales[..., 1] = np.where(n % 4 == 0, 2.0 ** -9, 2.0 ** -90)
    st.raw = ref.pack(codes, scales, D)
    st.cache = dev(st.raw)
    shared_check(tt, st, 4, [(0, seqs, 384)], scale=0.02)


@pytest.mark.parametrize("D,seqs", [(128, 3), (128, 70), (64, 4), (256, 3)])
def test_scores_that_rise_from_token_to_token(tt, D, seqs):
    """The reference moves in every step, inside a block and between the first and second half of a step."""
    st = Step(114, D, 1, 32, [330] * seqs, [1] * seqs)
    share(st, [(0, seqs, 320)])
    codes, scales = ref.unpack(st.raw, D)
    scales[..., 0], scales[..., 1] = 1.0, 2.0 ** -5
    codes[0] = 0
    for t in range(331):
        at = st.table[:, t // 32], slice(None), t % 32 // 16, t % 16
        codes[0][at[0], :, at[2], at[3], 0] = t // 4
    st.raw = ref.pack(codes, scales, D)
    st.cache = dev(st.raw)
    q = np.zeros((seqs, 4, D), np.float16)
    q[..., 0] = [1, 3, -2, 0.1]
    shared_check(tt, st, 4, [(0, seqs, 320)], scale=0.9, q=q)


def test_nan_in_the_shared_tokens_and_beside_them(tt):
    st = Step(115, 64, 2, 16, [200, 210, 70], [1] * 3)
    share(st, [(0, 2, 192)])
    codes, scales = ref.unpack(st.raw, 64)
    scales[st.table[0, 2], 0, 0, 0] = np.nan   # a shared key block of head 0
    scales[st.table[0, 3], 1, 0, 1] = np.nan   # a shared value block of head 1
    scales[st.table[2, 1], 0, 0, 1] = np.nan   # of the sequence that is in no group, seen
    st.raw = ref.pack(codes, scales, 64)
    st.cache = dev(st.raw)
    out = shared_check(tt, st, 4, [(0, 2, 192)]).cpu().numpy()
    assert np.isnan(out[:2]).all() and np.isnan(out[2, :2]).all() and np.isfinite(out[2, 2:]).all()
    q = st.rng.standard_normal((3, 4, 64)).astype(np.float16)
    st2 = Step(116, 64, 2, 16, [200, 210, 205], [1] * 3)
    q[1, 2, 5], q[2, 0, 1] = np.nan, np.inf   # a query that is not finite stays alone
    out = shared_check(tt, st2, 4, [(0, 3, 192)], q=q).cpu().numpy()
    bad = np.zeros((3, 4), bool)
    bad[1, 2] = bad[2, 0] = True
    assert np.array_equal(np.isnan(out).all(-1), bad) and np.isfinite(out[~bad]).all()


def test_in_place_and_rows_that_lie_apart(tt):
    st = Step(117, 128, 2, 32, [300, 290, 350], [1, 2, 1])
    start, shared = share(st, [(0, 3, 288)])
    wide = torch.randn((4, 12, 128), device="cuda").half()
    ws = tt.tetra_kv_shared_workspace(128, 4, 8, 2, 1)
    want = tt.tetra_kv_attend_shared(wide[:, :8].contiguous(), *st.args(), start, shared, torch.empty((4, 8, 128), dtype=torch.float16, device="cuda"), ws)
    apart = tt.tetra_kv_attend_shared(wide[:, :8], *st.args(), start, shared, torch.empty_like(want), ws)
    q = wide[:, :8].contiguous()
    assert tt.tetra_kv_attend_shared(q, *st.args(), start, shared, q, ws) is q
    assert torch.equal(want, apart) and torch.equal(want, q)


def test_long_prompts(tt):
    """Parts of many steps, two waves of them, and the attention that shares nothing."""
    for D, H, heads, seqs, shared in ((128, 8, 32, 6, 9000), (128, 2, 40, 24, 5000), (64, 1, 8, 3, 40000), (256, 4, 8, 2, 6000)):
        st = Step(118, D, H, 64, [shared + 5 * i for i in range(seqs)], [1] * seqs, width=shared // 64 + 4)
        start, tokens = share(st, [(0, seqs, shared - shared % 64)])
        q = torch.randn((seqs, heads, D), device="cuda").half()
        one = tt.tetra_kv_attend_shared(q, *st.args(), start, tokens, torch.empty_like(q), tt.tetra_kv_shared_workspace(D, seqs, heads, H, 1))
        two = tt.tetra_kv_attend(q, *st.args(), torch.empty_like(q), tt.tetra_kv_workspace(D))
        # No value is above 127 / 8.  Either output is off by 2^-11 of that for its own rounding, as much for the weights', and
        # (n / 16 + 64) 2^-23, for 40000 tokens 2^-11.7, for the sum's; for the scores (step_reference.attend) by 2 (D + 16) 2^-23 |q k| scale,
        # no more than 2^-11 where |q k| scale is below 7, which a standard normal q of 64 to 256 dims against values below 16 of mean square 9
        # passes by chance alone: |q k| scale < 9 * 4 even so, 2^-9.4.  Twice the sum: 2 (2^-11 + 2^-11 + 2^-11.7 + 2^-9.4) < 2^-7.
        assert (one.float() - two.float()).abs().max() <= 2.0 ** -7 * 127 / 8


def test_offsets_that_pass_32_bits(tt):
    """A cache of 4.6 GB; the shared pages live at its end."""
    D, H, P, pages = 128, 8, 128, 17600
    st = Step(119, D, H, P, [300, 280, 310], [1] * 3)
    start, shared = share(st, [(0, 3, 256)])
    cache = torch.empty((pages, H, P // 16, 32 * D + 16), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32
    moved = pages - 1 - st.table
    raw = torch.from_numpy(st.raw).cuda()
    for old, new in zip(st.table.reshape(-1), moved.reshape(-1)):
        cache[new] = raw[old]
    q = torch.randn((3, 32, D), device="cuda").half()
    ws = tt.tetra_kv_shared_workspace(D, 3, 32, H, 1)
    small = tt.tetra_kv_attend_shared(q, *st.args(), start, shared, torch.empty_like(q), ws)
    big = tt.tetra_kv_attend_shared(q, cache, wide(st, moved), st.d_starts, st.d_lengths, start, shared, torch.empty_like(q), ws)
    assert torch.equal(small, big)


@pytest.mark.parametrize("D,heads,H,rows,shared", [(128, 32, 8, [3000, 2500], 4096), (64, 16, 8, [3000, 1, 1500], 1024), (256, 16, 4, [900, 1100], 1024)])
def test_prompts_behind_prompts(tt, D, heads, H, rows, shared):
    """More items than parts, several of a CTA: against tetra_kv_attend, of which the sums and the weights' roundings are another's of the same bounds
    (two of 2^-11 of the mean of |v| a weight, one of 2^-11 of the result each)."""
    st = Step(125, D, H, 64, [shared + 5] * len(rows), rows)
    start, tokens = share(st, [(0, len(rows), shared)])
    q = torch.randn((st.total, heads, D), device="cuda").half()
    out = tt.tetra_kv_attend_shared(q, *st.args(), start, tokens, torch.empty_like(q), tt.tetra_kv_shared_workspace(D, st.total, heads, H, 1))
    want = tt.tetra_kv_attend(q, *st.args(), torch.empty_like(q), tt.tetra_kv_workspace(D))
    k, v = (torch.empty((shared, H, D), dtype=torch.float16, device="cuda") for _ in range(2))
    tt.tetra_kv_read(st.cache, st.d_table[:1], i32([0, shared]), i32([0]), k, v)
    most = v.float().abs().max()
    assert (out.float() - want.float()).abs().max() <= 2 * 2.0 ** -11 * most + 2 * 2.0 ** -11 * want.float().abs().max()


# ---- streams, graphs, refusals -----------------------------------------------------------------------------------------
def test_a_captured_call_follows_lengths_groups_and_pages(tt):
    """One graph, replayed with other groups, lengths, pages and queries; eager calls use its workspace in between."""
    D, H, heads, n = 128, 2, 8, 6
    st = Step(120, D, H, 16, [400] * n, [1] * n, width=40)
    start, shared, table = i32([0, 3, 6]), i32([0, 0]), wide(st, st.table)
    rows, lengths = st.d_starts, torch.zeros_like(st.d_lengths)
    q, out, ws = torch.zeros((n, heads, D), dtype=torch.float16, device="cuda"), torch.zeros((n, heads, D), dtype=torch.float16, device="cuda"), tt.tetra_kv_shared_workspace(D, n, heads, H, 2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        tt.tetra_kv_attend_shared(q, st.cache, table, rows, lengths, start, shared, out, ws)
    rng = np.random.default_rng(121)
    for split, tokens, before in (([0, 3, 6], [320, 160], [330, 340, 320, 200, 161, 160]), ([0, 6, 6], [128, 0], [128, 600, 130, 129, 400, 500]),
                                  ([0, 0, 0], [9, 9], [5] * 6), ([1, 3, 5], [512, 384], [7, 520, 513, 400, 385, -1])):
        st.table = rng.permutation(st.pages)[:n * st.width].reshape(n, st.width)
        new_start, new_shared = share(st, list(zip(split, split[1:], tokens)))
        for to, x in ((start, new_start), (shared, new_shared), (table, wide(st, st.table)), (lengths, i32(before + [0] * (len(lengths) - n))), (q, torch.randn((n, heads, D), device="cuda").half())):
            to.copy_(x)
        graph.replay()
        replayed = out.clone()
        eager = tt.tetra_kv_attend_shared(q, st.cache, table, rows, lengths, start, shared, torch.zeros_like(q), ws)
        assert torch.equal(replayed.view(torch.int16), eager.view(torch.int16))
        plain, bound = ref.attend(st.plain(), q.cpu().numpy(), st.table, st.starts, before, 1 / np.sqrt(D))
        assert (np.abs(replayed.cpu().numpy() - plain) <= 3 * bound).all()


def test_two_streams_with_workspaces_of_their_own(tt):
    st = Step(122, 128, 2, 64, [3000, 3010, 2999], [1] * 3)
    start, shared = share(st, [(0, 3, 2944)])
    q = torch.randn((3, 8, 128), device="cuda").half()
    new = lambda: tt.tetra_kv_shared_workspace(128, 3, 8, 2, 1)  # noqa: E731
    want = tt.tetra_kv_attend_shared(q, *st.args(), start, shared, torch.empty_like(q), new())
    streams, ws, outs = [torch.cuda.Stream() for _ in range(2)], [new(), new()], [[torch.empty_like(q) for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                tt.tetra_kv_attend_shared(q, *st.args(), start, shared, outs[k][i], ws[k])
    torch.cuda.synchronize()
    for o in outs[0] + outs[1]:
        assert torch.equal(o, want)
    other = torch.empty_like(q)
    tt.tetra_kv_attend_shared(q, *st.args(), start, shared, other, ws[0], stream=streams[1])
    streams[1].synchronize()
    assert torch.equal(other, want)


def test_a_workspace_for_more_serves_less(tt):
    st = Step(123, 64, 2, 16, [300, 320], [1, 1])
    start, shared = share(st, [(0, 2, 288)])
    q = torch.randn((2, 4, 64), device="cuda").half()
    ws = tt.tetra_kv_shared_workspace(64, 100, 16, 2, 10)
    ws.fill_(0xFF)  # but for tetra_kv_attend's counters, what is there does not matter
    ws[:4608] = 0
    a = tt.tetra_kv_attend_shared(q, *st.args(), start, shared, torch.empty_like(q), ws)
    b = tt.tetra_kv_attend_shared(q, *st.args(), start, shared, torch.empty_like(q), tt.tetra_kv_shared_workspace(64, 2, 4, 2, 1))
    assert torch.equal(a, b)


def test_the_binding_refuses(tt):
    st = Step(124, 128, 2, 32, [400, 400], [1, 1])
    start, shared = share(st, [(0, 2, 384)])
    h, ws = torch.zeros((2, 4, 128), dtype=torch.float16, device="cuda"), tt.tetra_kv_shared_workspace(128, 2, 4, 2, 1)
    c = tt.tetra_kv_attend_shared

    def refused(match, *args, **more):
        with pytest.raises(tt.TetraError, match=match):
            c(*args, **more)
    refused("q: Float", h.float(), *st.args(), start, shared, h, ws)
    refused("group_start: wrong", h, *st.args(), start[:1], shared, h, ws)
    refused("group_start: Long", h, *st.args(), start.long(), shared, h, ws)
    refused("shared: Float", h, *st.args(), start, shared.float(), h, ws)
    refused("shared: tensor is not on", h, *st.args(), start, shared.cpu(), h, ws)
    refused("out: wrong", h, *st.args(), start, shared, h[:1], ws)
    refused("buffer too small", h, *st.args(), start, shared, h, ws[:-1])
    refused("buffer too small", h, *st.args(), start, shared, h, tt.tetra_kv_workspace(128))
    refused("out of range", h, *st.args(), start, shared, h, ws, float("inf"))
    many = torch.zeros(1026, dtype=torch.int32, device="cuda")
    refused("out of range", h, *st.args(), many, many[:1025].contiguous(), h, ws)
    none = torch.zeros((0, 4, 128), dtype=torch.float16, device="cuda")
    assert c(none, *st.args(), start, shared, none, ws) is none
