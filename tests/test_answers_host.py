"""Rows at given positions, attention of groups and log probabilities without a GPU: what the C entries refuse, sizes, and how their
kernels are ordered."""
import ctypes as C

import numpy as np
import pytest
import torch

import test_launch_order_source as order
from test_step_host import BAD_VIEWS, tt, view  # noqa: F401


@pytest.mark.parametrize("change,rc", BAD_VIEWS)
def test_a_bad_cache(tt, change, rc):  # noqa: F811
    L, c = tt.lib(), view(tt, **change)
    p = c.keep[0].data_ptr() + 255 & ~255
    r = tt.KvRows(k=p, v=p, k_stride=256, v_stride=256, rows=1, eps=1e-6, inv_freq=p)
    a = tt.KvAxes(positions=p, axis=p, stride=3, axes=3)
    g = tt.KvGroups(group_start=p, shared=p, groups=1)
    assert L.tetra_kv_append_at(C.byref(c), C.byref(r), C.byref(a), None) == rc
    assert L.tetra_kv_attend_shared(C.byref(c), C.byref(g), p, 512, p, 1, 4, 1.0, p, 1 << 30, None) == rc


@pytest.mark.parametrize("change,rc", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(inv_freq=None), -1), (dict(rows=-1), -2), (dict(rows=65537), -2),
    (dict(k_stride=255), -2), (dict(v_stride=255), -2), (dict(q_stride=511), -2), (dict(q_heads=5), -2), (dict(q_heads=0), -2), (dict(q_heads=4098), -2),
    (dict(half_type=2), -2), (dict(half_type=-1), -2), (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2),
    (dict(q=258), -3), (dict(k=257), -3), (dict(v=258), -3), (dict(q_out=257), -3), (dict(inv_freq=260), -3), (dict(q_weight=258), -3), (dict(k_weight=257), -3),
    (dict(positions=None), -1), (dict(axis=None), -1), (dict(axes=0), -2), (dict(axes=9), -2), (dict(axes=-1), -2), (dict(stride=2), -2), (dict(positions=258), -3), (dict(rows=0), 0)])
def test_append_at_refuses(tt, change, rc):  # noqa: F811
    L, c = tt.lib(), view(tt)
    f = dict(q=256, k=256, v=256, q_out=256, q_stride=512, k_stride=256, v_stride=256, rows=1, q_heads=4, eps=1e-6, inv_freq=256, positions=256, axis=257, stride=3, axes=3)
    f.update(change)
    a = tt.KvAxes(**{k: f.pop(k) for k in ("positions", "axis", "stride", "axes")})
    assert L.tetra_kv_append_at(C.byref(c), C.byref(tt.KvRows(**f)), C.byref(a), None) == rc
    assert L.tetra_kv_append_at(C.byref(c), None, C.byref(a), None) == -1
    assert L.tetra_kv_append_at(C.byref(c), C.byref(tt.KvRows(**f)), None, None) == -1


def test_attend_shared_refuses(tt):  # noqa: F811
    L, c = tt.lib(), view(tt)
    need = lambda groups: L.tetra_kv_shared_workspace_bytes(128, 1, 4, 2, groups)  # noqa: E731
    good = dict(q=256, stride=512, out=256, rows=1, heads=4, scale=0.1, ws=256, n=need(2), start=256, shared=256, groups=2)
    for change, rc in ((dict(q=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(start=None), -1), (dict(shared=None), -1), (dict(groups=-1), -2), (dict(groups=1025), -2),
                       (dict(start=258), -3), (dict(shared=257), -3), (dict(heads=3), -2), (dict(heads=0), -2), (dict(heads=4098, stride=4098 * 128), -2),
                       (dict(stride=504), -2), (dict(stride=516), -3), (dict(q=264), -3), (dict(out=264), -3), (dict(ws=272), -3), (dict(n=need(2) - 1), -6),
                       (dict(groups=0, start=None, shared=None, n=need(0) - 1), -6), (dict(scale=float("inf")), -2), (dict(scale=float("nan")), -2), (dict(scale=2.4e38), -2),
                       (dict(rows=65537), -2), (dict(rows=-1), -2), (dict(rows=0), 0)):
        a = dict(good, **change)
        g = tt.KvGroups(group_start=a["start"], shared=a["shared"], groups=a["groups"])
        got = L.tetra_kv_attend_shared(C.byref(c), C.byref(g), a["q"], a["stride"], a["out"], a["rows"], a["heads"], a["scale"], a["ws"], a["n"], None)
        assert got == rc, change
    assert L.tetra_kv_attend_shared(C.byref(c), None, 256, 512, 256, 1, 4, 0.1, 256, 1 << 30, None) == -1


def test_the_workspace_of_groups(tt):  # noqa: F811
    L = tt.lib()
    size = L.tetra_kv_shared_workspace_bytes
    for bad in ((96, 1, 4, 2, 1), (128, -1, 4, 2, 1), (128, 65537, 4, 2, 1), (128, 1, 5, 2, 1), (128, 1, 0, 1, 1), (128, 1, 4098, 2, 1), (128, 1, 4, 0, 1), (128, 1, 1025, 1025, 1), (128, 1, 4, 2, -1),
                (128, 1, 4, 2, 1025)):
        assert size(*bad) == 0, bad
        with pytest.raises(tt.TetraError, match="rejected"):
            tt.tetra_kv_shared_workspace(*bad, device="cpu")
    for D in (64, 128, 256):
        for kv in (1, 8):
            made = [size(D, rows, heads, kv, groups) for rows in (0, 1, 64, 65536) for heads in (8, 64) for groups in (0, 1, 1024)]
            assert all(n >= L.tetra_kv_workspace_bytes(D) for n in made)
            # more of any takes no less
            for i, (r, h, g) in enumerate((r, h, g) for r in range(4) for h in range(2) for g in range(3)):
                for step, there in ((6, r < 3), (3, h < 1), (1, g < 2)):
                    assert not there or made[i + step] >= made[i], (D, kv, r, h, g)
    assert tt.tetra_kv_shared_workspace(128, 1, 4, 2, 1, device="cpu").numel() == size(128, 1, 4, 2, 1)


def test_logprobs_refuses(tt):  # noqa: F811
    L = tt.lib()
    good = dict(logits=256, temperature=256, tokens=256, logprob=256, rank=256, entropy=256, top_tokens=256, top_logprob=256, row_stride=100, rows=1, vocab=100, given=3, top=5)
    for change, rc in ((dict(logits=None), -1), (dict(tokens=None), -1), (dict(logprob=None), -1), (dict(top_tokens=None), -1), (dict(top_logprob=None), -1), (dict(rows=-1), -2), (dict(rows=65536), -2),
                       (dict(vocab=0), -2), (dict(vocab=(1 << 24) + 1, row_stride=1 << 25), -2), (dict(row_stride=99), -2), (dict(half_type=2), -2), (dict(half_type=-1), -2),
                       (dict(given=-1), -2), (dict(given=65), -2), (dict(top=-1), -2), (dict(top=33), -2), (dict(logits=258), -3), (dict(temperature=258), -3), (dict(tokens=257), -3),
                       (dict(logprob=258), -3), (dict(rank=258), -3), (dict(entropy=257), -3), (dict(top_tokens=258), -3), (dict(top_logprob=258), -3), (dict(half_type=1, logits=257), -3),
                       (dict(rows=0), 0)):
        assert L.tetra_logprobs(C.byref(tt.LogprobsRows(**dict(good, **change))), None) == rc, change
    assert L.tetra_logprobs(None, None) == -1


def test_the_binding_wants_tensors_on_the_device(tt):  # noqa: F811
    f, i = torch.zeros((1, 100)), torch.zeros((1, 2), dtype=torch.int32)
    with pytest.raises(tt.TetraError, match="logits: tensor is not on the device"):
        tt.tetra_logprobs(f, i, f[:, :2])
    with pytest.raises(tt.TetraError, match="logits: Double"):
        tt.tetra_logprobs(f.double(), i, f[:, :2])
    cache = torch.zeros((2, 2, 1, 32 * 64 + 16), dtype=torch.uint8)
    h = torch.zeros((1, 2, 64), dtype=torch.float16)
    with pytest.raises(tt.TetraError, match="cache: tensor is not on the device"):
        tt.tetra_kv_append_at(None, h, h, cache, i, i[0], i[0, :1], i, torch.zeros(32, dtype=torch.uint8), None, torch.zeros(32, dtype=torch.float64))
    with pytest.raises(tt.TetraError, match="cache: tensor is not on the device"):
        tt.tetra_kv_attend_shared(h, cache, i, i[0], i[0, :1], i[0], i[0, :1], h, cache)


# ---- order ---------------------------------------------------------------------------------------------------------------
def test_every_kernel_waits_before_it_touches_memory():
    """All that these kernels read or write comes behind their wait, and what they release waits too."""
    text = dict(order.sources())
    for f in ("kv_append_at.cu", "kv_prefix.cu", "logprobs.cu"):
        assert text[f].count("pdl_wait();") >= 1, f
        assert text[f].count("pdl_release();") <= text[f].count("pdl_wait();"), f
    for name, (params, body) in order.KERNELS.items():
        if name in ("k_kv_append_at", "k_kv_append_blocks", "k_kv_prefix", "k_kv_join", "k_logprobs"):
            before = body[:body.index("pdl_wait")] if "pdl_wait" in body else ""
            assert "page_table" not in before and "row_start" not in before, name


def test_the_kernels_of_answers_are_found():
    assert {"k_kv_append_at", "k_kv_append_blocks", "k_kv_prefix", "k_kv_join", "k_logprobs"} <= set(order.KERNELS)
