"""Scores so large that float32 has no fractions of them: the weights go by the differences of scores, which are exact.

A query is 16384 in 16 dims and 1 in the last one, a key 64 in those and a code c in the last: the score in powers of two is
(2^24 + c) 2^j, exactly, where scale log2(e) is one in float32 (its products and sums are whole numbers that float32 holds)."""
import numpy as np
import pytest
import torch

import step_reference as ref
from test_gpu_kv import Step, dev

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(np.log(2.0)))


def test_the_scale_is_one_in_powers_of_two():
    assert np.float32(SCALE) * np.float32(1.4426950408889634) == np.float32(1)


# j: float32's step at 2^(24 + j) is 2^(j + 1).  A CTA to an item, wide tiles, a warp to an item.
@pytest.mark.parametrize("j", range(8))
@pytest.mark.parametrize("before,rows", [([16 * 8 * 5 - 1], [1]), ([16 * 8 * 3 - 16], [16]), ([70] * 160, [1] * 160)])
def test_scores_without_fractions(before, rows, j):
    from paper_2609_35465_b200 import tetra
    D, H = 64, 2
    st = Step(61, D, H, 64, before, rows)
    codes, scales = ref.unpack(st.raw, D)
    values = codes[1].copy()
    q = torch.zeros((st.total, 4, D), dtype=torch.float16, device="cuda")
    q[..., :16], q[..., D - 1] = 16384, 1
    ws = tetra.tetra_kv_workspace(D)
    for by in (0, 2, 4, 14, 16, 40):  # what c grows by with every eighth block, a warp's next
        for lv in (-24, -16, -8, 0, 3, 8):  # log2 of the values' scale
            codes[0] = 0
            codes[0, ..., :16] = 64
            for s, b in enumerate(before):
                for block in range((b + rows[s] + 15) // 16):
                    codes[0, st.table[s, block // 4], :, block % 4, :, D - 1] = min(126, block // (8 if len(before) == 1 else 1) * by)
            codes[1] = np.rint(values / 127) if lv == 8 else values  # values that float16 holds
            scales[..., 0], scales[..., 1] = 2.0 ** j, 2.0 ** lv
            st.raw = ref.pack(codes, scales, D)
            st.cache = dev(st.raw)
            out = tetra.tetra_kv_attend(q, *st.args(), torch.full_like(q, 7.5), ws, SCALE).cpu().numpy().astype(np.float64)
            plain = st.plain()
            for s in (range(len(before)) if len(before) < 9 else (0, 77, 159)):
                kv, _ = plain.tokens(st.table, s, before[s] + rows[s])
                for i in range(rows[s]):
                    n = before[s] + i + 1
                    x = kv[0, :n, 0, D - 1]  # c 2^j; what the scores have alike drops out
                    p = np.exp2(x - x.max())
                    p /= p.sum()
                    v = kv[1, :n].repeat(2, 1)
                    want, size = np.einsum("p,phd->hd", p, v), np.einsum("p,phd->hd", p, np.abs(v))
                    # The output is rounded once.  40 additions of 2^-24 at most, above and below the division, and the scale's own
                    # rounding: 2^-17.  A weight times scale is a power of two, exact in float16 down to 2^-24 and off by 2^-25
                    # at most below that; the largest of a column is 2^E, E >= min(lv, -8): its reference is rounded
                    # to a step of the scores, by eight at most where the steps are 16, and where they are larger it is the score itself.
                    E = min(lv, -8)
                    lost = (p < p.max() * 2.0 ** (-24 - E)).sum() * 2.0 ** (-25 - E) * 127 * 2.0 ** lv * p.max()
                    bound = 2.0 ** -11 * np.abs(want) + 2.0 ** -17 * size + lost + 2.0 ** -25
                    assert (np.abs(out[st.starts[s] + i] - want) <= bound).all(), (by, lv, s, i)
