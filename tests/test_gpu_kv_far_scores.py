"""Scores of any finite size: a row that sees a token has an output from its tokens' values, however far below zero all of its scores lie."""
import numpy as np
import pytest
import torch

import step_reference as ref
from test_gpu_kv import Step, dev

pytestmark = pytest.mark.gpu


def far_step(seed, D, H, P, before, rows, log_scale, own):
    """Keys that are alike (code -127 in every dim) but those of each sequence's third token, whose code is `own`."""
    st = Step(seed, D, H, P, before, rows)
    codes, scales = ref.unpack(st.raw, D)
    codes[0] = -127
    for s in range(len(before)):
        codes[0, st.table[s, 0], :, 0, 2] = own
    scales[..., 0] = 2.0 ** log_scale
    st.raw = ref.pack(codes, scales, D)
    st.cache = dev(st.raw)
    return st


@pytest.mark.parametrize("D,H,heads", [(128, 2, 8), (64, 1, 5), (256, 1, 2)])
@pytest.mark.parametrize("before,rows", [([40], [1]), ([9000, 5], [1, 1]), ([300, 5], [16, 2]), ([3] * 64, [1] * 64)])
@pytest.mark.parametrize("log_scale", [70, 97, 112])
def test_scores_far_below_zero(before, rows, D, H, heads, log_scale):
    """One token's score is the largest by far: the output is its value, exactly (a float16 number).  Where all are alike the
    weights are, too: the output is the mean of the values."""
    from paper_2609_35465_b200 import tetra
    for own in (-1, -127):
        st = far_step(60, D, H, 16, before, rows, log_scale, own)
        q = torch.ones((st.total, heads, D), dtype=torch.float16, device="cuda")
        out = tetra.tetra_kv_attend(q, *st.args(), torch.full_like(q, 7.5), tetra.tetra_kv_workspace(D)).cpu().numpy().astype(np.float64)
        plain = st.plain()
        for s, (b, n) in enumerate(zip(before, rows)):
            v = plain.tokens(st.table, s, b + n)[0][1].repeat(heads // H, 1)  # [tokens, heads, D]
            for i in range(n):
                have = out[st.starts[s] + i]
                if own == -1:
                    assert np.array_equal(have, v[2]), (s, i)
                else:
                    # equal weights are exact in float16 (a power of two); sums are float32: 2^-24 of the sum of sizes for each
                    # addition; the output is rounded once
                    seen = v[:b + i + 1]
                    want, size = seen.mean(0), np.abs(seen).mean(0)
                    assert (np.abs(have - want) <= 2.0 ** -11 * np.abs(want) + (b + n + 32) * 2.0 ** -24 * size + 2.0 ** -25).all(), (s, i)
