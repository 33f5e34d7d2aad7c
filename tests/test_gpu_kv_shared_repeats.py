"""Attention of groups again and again, each call on an idle GPU: the same bits every time, whatever the waits and the instruction
caches of a call are like.  (A column's sums read ahead of their last products showed once in about a thousand such calls.)"""
import numpy as np
import pytest
import torch

from test_gpu_kv import Step, dev
from test_gpu_kv_shared import share, tt  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,heads,shared,rows,seed", [(128, 32, 1488, [5, 11, 10, 11, 5], 1), (128, 32, 320, [1, 1], 2), (64, 16, 1008, [9, 9, 9], 3), (256, 16, 704, [20, 13], 4)])
def test_the_same_bits_every_time(tt, D, heads, shared, rows, seed):  # noqa: F811
    st = Step(300 + seed, D, 8, 16, [shared + 2] * len(rows), rows)
    start, tokens = share(st, [(0, len(rows), shared)])
    q = dev(st.rng.standard_normal((st.total, heads, D)).astype(np.float16))
    ws = tt.tetra_kv_shared_workspace(D, st.total, heads, st.H, 1)
    want = tt.tetra_kv_attend_shared(q, *st.args(), start, tokens, torch.empty_like(q), ws).clone()
    out, other = torch.empty_like(q), torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(12000):
        torch.cuda.synchronize()
        tt.tetra_kv_attend_shared(q, *st.args(), start, tokens, out, ws)
        other += (out != want).any()
    assert int(other) == 0
