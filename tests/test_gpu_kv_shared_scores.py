"""Attention of groups: scores that float32 has no fractions of, scores far below zero, and values that are zero where the scores are largest.

A key block's scale is no power of two here: score times scale is rounded, and what is rounded is what the weights go by."""
import numpy as np
import pytest
import torch

import step_reference as ref
from shared_cut import cut
from test_gpu_kv import Step, dev
from test_gpu_kv_large_scores import SCALE
from test_gpu_kv_shared import share, shared_check, tt  # noqa: F401

pytestmark = pytest.mark.gpu


def attended(tt, st, q, shared, scale):  # noqa: F811
    start, tokens = share(st, [(0, len(st.before), shared)])
    ws = tt.tetra_kv_shared_workspace(st.D, st.total, q.shape[1], st.H, 1)
    return tt.tetra_kv_attend_shared(q, *st.args(), start, tokens, torch.full_like(q, 7.5), ws, scale).cpu().numpy().astype(np.float64)


# float32's step at 2^(24 + j) is 2^(j + 1).  One slot's columns and both's.
@pytest.mark.parametrize("j", [0, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("D,seqs,rows", [(64, 3, 2), (128, 40, 1), (128, 3, 1), (256, 5, 1), (64, 70, 1)])
def test_scores_without_fractions(tt, D, seqs, rows, j):  # noqa: F811
    """As in test_gpu_kv_large_scores: a query is 16384 in 16 dims and 1 in the last one, a key 64 in those and an even code c in the last."""
    shared = 640
    st = Step(501, D, 1, 64, [shared + i % 7 for i in range(seqs)], [rows] * seqs)
    share(st, [(0, seqs, shared)])
    codes, scales = ref.unpack(st.raw, D)
    values = codes[1].copy()
    q = torch.zeros((st.total, 4, D), dtype=torch.float16, device="cuda")
    q[..., :16], q[..., D - 1] = 16384, 1
    for times in (1.37, 1.9):
        for by in (0, 2, 40):  # what c grows by with every fifth block
            for lv in (-24, -12, 8):
                codes[0] = 0
                codes[0, ..., :16] = 64
                for block in range(-(-(shared + 10) // 16)):
                    codes[0, st.table[:, block // 4], :, block % 4, :, D - 1] = min(126, block // 5 * by)
                codes[1] = np.rint(values / 127) if lv == 8 else values  # values that float16 holds
                scales[..., 0], scales[..., 1] = times * 2.0 ** j, 2.0 ** lv
                st.raw = ref.pack(codes, scales, D)
                st.cache = dev(st.raw)
                out = attended(tt, st, q, shared, SCALE)
                assert np.isfinite(out).all(), (times, by, lv)
                alone = tt.tetra_kv_attend(q, *st.args(), torch.full_like(q, 7.5), tt.tetra_kv_workspace(D), SCALE).cpu().numpy().astype(np.float64)
                plain = st.plain()
                for s in (0, 1, seqs - 1):
                    n = st.before[s] + rows
                    kv, _ = plain.tokens(st.table, s, n)
                    c = np.rint(kv[0, :, 0, D - 1] / np.float64(np.float32(times * 2.0 ** j)))
                    x = (np.float32(2.0 ** 24) + c.astype(np.float32)) * np.float32(times * 2.0 ** j)  # rounded: whole numbers
                    for i in range(rows):
                        seen = st.before[s] + i + 1
                        d = x[:seen].astype(np.float64)
                        p = np.exp2(d - d.max())
                        p /= p.sum()
                        v = kv[1, :seen].repeat(4, 1)
                        want, size = np.einsum("p,phd->hd", p, v), np.einsum("p,phd->hd", p, np.abs(v))
                        # The output is rounded once; sums are (n / 16 + 64) 2^-23 of the mean of |v| off at most (test_gpu_kv_shared),
                        # 2^-16.  A weight times scale is a power of two, exact in float16 down to 2^-24 and off by 2^-25 at most below that;
                        # the largest of a column is 2^E, E >= min(lv, -8): its reference is rounded to a step of the scores, by
                        # eight at most where the steps are 16, and where they are larger it is the score itself.
                        E = min(lv, -8)
                        lost = (p < p.max() * 2.0 ** (-24 - E)).sum() * 2.0 ** (-25 - E) * 127 * 2.0 ** lv * p.max()
                        bound = 2.0 ** -11 * np.abs(want) + 2.0 ** -16 * size + lost + 2.0 ** -25
                        for have in (out, alone):
                            assert (np.abs(have[st.starts[s] + i] - want) <= bound).all(), (times, by, lv, s, i)


@pytest.mark.parametrize("D,heads,seqs", [(128, 8, 3), (64, 5, 40), (256, 2, 4), (128, 4, 70)])
@pytest.mark.parametrize("log_scale", [20, 27, 70, 97, 112])
@pytest.mark.parametrize("times", [1.0, 1.37])
def test_scores_far_below_zero(tt, D, heads, seqs, log_scale, times):  # noqa: F811
    """One token's score is the largest by far: the output is its value, exactly.  Where all are alike: the mean."""
    shared = 448
    for own in (-1, -127):
        st = Step(502, D, 1, 16, [shared + i % 3 for i in range(seqs)], [1] * seqs)
        share(st, [(0, seqs, shared)])
        codes, scales = ref.unpack(st.raw, D)
        codes[0] = -127
        codes[0, st.table[0, 9], :, 0, 2] = own
        scales[..., 0] = times * 2.0 ** log_scale
        st.raw = ref.pack(codes, scales, D)
        st.cache = dev(st.raw)
        q = torch.ones((st.total, heads, D), dtype=torch.float16, device="cuda")
        out, plain = attended(tt, st, q, shared, None), st.plain()
        for s in (0, 1, seqs - 1):
            v = plain.tokens(st.table, s, st.before[s] + 1)[0][1].repeat(heads, 1)
            if own == -1:
                assert np.array_equal(out[s], v[9 * 16 + 2]), s
            else:
                # equal weights are powers of two, exact in float16; sums as above
                want, size = v.mean(0), np.abs(v).mean(0)
                assert (np.abs(out[s] - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -16 * size + 2.0 ** -25).all(), s


@pytest.mark.parametrize("D,seqs,group,cases", [(128, 3, 2, 12), (128, 9, 16, 2), (64, 2, 2, 12), (256, 2, 2, 5)])
def test_values_of_zero_under_the_largest_scores(tt, D, seqs, group, cases):  # noqa: F811
    """Blocks of ordinary values set a reference; blocks of zeros, or of next to nothing, have a token each so many powers of two above it;
    then come blocks of ordinary values, as much above or below that.  The prompt is 512 such tokens again and again, so that each of the
    parts that it is cut into has all of them."""
    heads, times = 8, 18
    ctas = torch.cuda.get_device_properties(0).multi_processor_count
    parts = cut(D, heads, group, [(seqs, 512 * times)], ctas)
    assert any(steps >= 6 for mine in parts for steps, _ in mine)
    st = Step(503, D, heads, 16, [512] * seqs, [1] * seqs)
    own = st.table[:, 32:]
    st.table = np.concatenate([np.tile(st.table[:1, :32], (seqs, times)), own], 1)
    st.width, st.before = st.table.shape[1], [512 * times + i % 3 for i in range(seqs)]
    block = st.table[0, :32]
    q = np.zeros((seqs, group * heads, D), np.float16)
    q[..., :2] = 1
    codes, scales = ref.unpack(st.raw, D)
    for above, last, log_value in [(a, b, v) for a in (127, 120) for b in (60, 10, -30) for v in (None, -100)][:cases]:
        codes[0] = 0
        codes[0, ..., 0] = -60                              # the reference is -67
        scales[..., 0], scales[..., 1] = 1.0, 1.0
        codes[0, block[8:24], :, 0, 5, 0] = above - 67      # both slots' steps
        scales[block[8:24], :, 0, 1] = 0.0 if log_value is None else 2.0 ** log_value
        codes[0, block[[24, 28]], :, 0, 3, 0], codes[0, block[[24, 28]], :, 0, 3, 1] = above - 67, last
        st.raw = ref.pack(codes, scales, D)
        st.cache = dev(st.raw)
        shared_check(tt, st, group * heads, [(0, seqs, 512 * times)], scale=SCALE, q=q)
