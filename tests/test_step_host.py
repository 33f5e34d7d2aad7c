"""The cache, its attention and the sampler without a GPU: what the calls refuse (in the binding and in the C ABI), sizes, and
the plain forms that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import step_reference as ref
from paper_2609_35465_b200 import build as tbuild


@pytest.fixture(scope="module")
def tt():
    tbuild.build()
    from paper_2609_35465_b200 import tetra
    return tetra


def test_cache_and_workspace_sizes(tt):
    L = tt.lib()
    assert L.tetra_kv_cache_bytes(3, 64, 8, 128) == 3 * 8 * 4 * (32 * 128 + 16)
    for shape in ((0, 64, 8, 128), (3, 0, 8, 128), (3, 24, 8, 128), (3, 64, 0, 128), (3, 64, 8, 80), (3, 64, 1025, 128), (3, (1 << 20) + 16, 8, 128), (-1, 64, 8, 128)):
        assert L.tetra_kv_cache_bytes(*shape) == 0, shape
        with pytest.raises(tt.TetraError, match="rejected"):
            tt.tetra_kv_cache(*shape, device="cpu")
    assert tt.tetra_kv_cache(3, 64, 8, 128, device="cpu").shape == (3, 8, 4, 32 * 128 + 16)
    assert all(L.tetra_kv_workspace_bytes(d) > 0 for d in (64, 128, 256)) and L.tetra_kv_workspace_bytes(96) == 0
    with pytest.raises(tt.TetraError, match="rejected"):
        tt.tetra_kv_workspace(96, device="cpu")


def address(t):
    return t.data_ptr()


def view(tt, D=128, **change):
    """A tetra_kv_cache of host memory: nothing here reaches a launch."""
    keep = [torch.zeros(1 << 16, dtype=torch.uint8) for _ in range(4)]
    at = [(address(t) + 255) & ~255 for t in keep]
    f = dict(cache=at[0], page_table=at[1], row_start=at[2], lengths=at[3], table_stride=4, pages=3, page_tokens=32, kv_heads=2, head_dim=D, seqs=2, width=4)
    f.update(change)
    c = tt.KvCache(**f)
    c.keep = keep
    return c


BAD_VIEWS = [(dict(cache=None), -1), (dict(page_table=None), -1), (dict(row_start=None), -1), (dict(lengths=None), -1),
             (dict(pages=0), -2), (dict(page_tokens=40), -2), (dict(kv_heads=0), -2), (dict(head_dim=96), -2), (dict(seqs=0), -2), (dict(seqs=1025), -2),
             (dict(width=0), -2), (dict(table_stride=3), -2), (dict(width=1 << 27, table_stride=1 << 27), -2)]


@pytest.mark.parametrize("change,rc", BAD_VIEWS)
def test_every_call_refuses_a_bad_cache(tt, change, rc):
    L, c = tt.lib(), view(tt, **change)
    p = c.keep[0].data_ptr() + 255 & ~255
    r = tt.KvRows(k=p, v=p, k_stride=256, v_stride=256, rows=1, eps=1e-6)
    assert L.tetra_kv_append(C.byref(c), C.byref(r), None) == rc
    assert L.tetra_kv_read(C.byref(c), p, p, 1, None) == rc
    assert L.tetra_kv_attend(C.byref(c), p, 512, p, 1, 4, 1.0, p, 1 << 30, None) == rc


def test_misaligned_views(tt):
    L = tt.lib()
    for name, by in (("cache", 8), ("page_table", 2), ("row_start", 2), ("lengths", 1)):
        c = view(tt)
        setattr(c, name, getattr(c, name) + by)
        assert L.tetra_kv_read(C.byref(c), 256, 256, 1, None) == -3, name


@pytest.mark.parametrize("change,rc", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(rows=-1), -2), (dict(rows=65537), -2),
    (dict(k_stride=255), -2), (dict(v_stride=255), -2), (dict(q_stride=511), -2), (dict(q_heads=5), -2), (dict(q_heads=0), -2), (dict(q_heads=4098), -2),
    (dict(half_type=2), -2), (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2), (dict(rows=0), 0),
    (dict(q=258), -3), (dict(k=257), -3), (dict(v=258), -3), (dict(q_out=257), -3), (dict(inv_freq=260), -3), (dict(q_weight=258), -3), (dict(k_weight=257), -3)])
def test_append_refuses(tt, change, rc):
    L, c = tt.lib(), view(tt)
    f = dict(q=256, k=256, v=256, q_out=256, q_stride=512, k_stride=256, v_stride=256, rows=1, q_heads=4, eps=1e-6)
    f.update(change)
    assert L.tetra_kv_append(C.byref(c), C.byref(tt.KvRows(**f)), None) == rc
    assert L.tetra_kv_append(C.byref(c), None, None) == -1


def test_read_and_attend_refuse(tt):
    L, c = tt.lib(), view(tt)
    assert L.tetra_kv_read(C.byref(c), None, 256, 1, None) == -1
    assert L.tetra_kv_read(C.byref(c), 256, 264, 1, None) == -3
    assert L.tetra_kv_read(C.byref(c), 256, 256, 0, None) == 0
    ws = L.tetra_kv_workspace_bytes(128)
    good = dict(q=256, stride=512, out=256, rows=1, heads=4, scale=0.1, ws=256, n=ws)
    for change, rc in ((dict(q=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(heads=3), -2), (dict(heads=0), -2), (dict(heads=4098, stride=4098 * 128), -2),
                       (dict(stride=504), -2), (dict(stride=516), -3), (dict(q=264), -3), (dict(out=264), -3), (dict(ws=272), -3), (dict(n=ws - 1), -6),
                       (dict(scale=float("inf")), -2), (dict(scale=float("nan")), -2), (dict(rows=65537), -2), (dict(rows=0), 0)):
        a = dict(good, **change)
        got = L.tetra_kv_attend(C.byref(c), a["q"], a["stride"], a["out"], a["rows"], a["heads"], a["scale"], a["ws"], a["n"], None)
        assert got == rc, change


def test_attend_refuses_a_scale_that_no_score_has(tt):
    """The kernel works in powers of two: the scale times log2(e) has to be finite as well."""
    L, c = tt.lib(), view(tt)
    for scale in (2.4e38, -2.4e38, float(np.finfo(np.float32).max)):
        assert L.tetra_kv_attend(C.byref(c), 256, 512, 256, 1, 4, scale, 256, L.tetra_kv_workspace_bytes(128), None) == -2
    assert L.tetra_kv_attend(C.byref(c), 256, 512, 256, 0, 4, 2.0 ** 127, 256, L.tetra_kv_workspace_bytes(128), None) == 0  # no rows, no launch


def test_sample_refuses(tt):
    L = tt.lib()
    good = dict(logits=256, u=256, tokens=256, row_stride=100, rows=1, vocab=100)
    for change, rc in ((dict(logits=None), -1), (dict(u=None), -1), (dict(tokens=None), -1), (dict(rows=-1), -2), (dict(rows=65536), -2), (dict(vocab=0), -2),
                       (dict(vocab=393217, row_stride=393217), -2), (dict(row_stride=99), -2), (dict(half_type=2), -2), (dict(half_type=-1), -2), (dict(rows=0), 0),
                       (dict(logits=258), -3), (dict(u=257), -3), (dict(temperature=258), -3), (dict(top_k=258), -3), (dict(top_p=258), -3), (dict(min_p=258), -3),
                       (dict(tokens=257), -3), (dict(prob=257), -3)):
        r = tt.SampleRows(**dict(good, **change))
        assert L.tetra_sample(C.byref(r), None) == rc, change
    assert L.tetra_sample(None, None) == -1


def test_the_binding_wants_tensors_on_the_device(tt):
    f = torch.zeros((1, 100))
    with pytest.raises(tt.TetraError, match="logits: tensor is not on the device"):
        tt.tetra_sample(f, f[0, :1], torch.zeros(1, dtype=torch.int32))
    with pytest.raises(tt.TetraError, match="logits: Double"):
        tt.tetra_sample(f.double(), f[0, :1], torch.zeros(1, dtype=torch.int32))
    cache = torch.zeros((2, 2, 1, 32 * 64 + 16), dtype=torch.uint8)
    i = torch.zeros(2, dtype=torch.int32)
    h = torch.zeros((1, 2, 64), dtype=torch.float16)
    with pytest.raises(tt.TetraError, match="cache: tensor is not on the device"):
        tt.tetra_kv_append(None, h, h, cache, i[None], i, i[:1], None)
    with pytest.raises(tt.TetraError, match="cache: Float"):
        tt.tetra_kv_read(cache.float(), i[None], i, i[:1], h, h)
    with pytest.raises(TypeError, match="expected a tensor"):
        tt.tetra_kv_attend(h, None, i[None], i, i[:1], h, cache)


# ---- the plain forms --------------------------------------------------------------------------------------------------
def test_records_are_a_bijection():
    for D in (64, 128, 256):
        places = np.concatenate([p.reshape(-1) for p in ref.byte_places(D)])
        assert np.array_equal(np.sort(places), np.arange(32 * D))
        rng = np.random.default_rng(D)
        raw = rng.integers(0, 256, (2, 3, 32 * D + 16)).astype(np.uint8)
        raw[..., 32 * D:] = 0
        codes, scales = ref.unpack(raw, D)
        assert np.array_equal(ref.pack(codes, scales, D), raw)


def test_least_scale():
    for amax, want in ((0.0, 0.0), (127.0, 1.0), (np.nextafter(127.0, 200), 2.0), (63.5, 0.5), (64.0, 1.0), (1.0, 2.0 ** -6), (2.0 ** -126, 2.0 ** -126), (2.0 ** -127, 0.0), (254.0, 2.0)):
        assert ref.least_scale(amax) == want


def test_a_cache_does_not_depend_on_the_cut_but_for_one_rounding():
    """37 tokens at once, one by one, or in pieces: equal scales; codes that differ by one at most where a scale grew."""
    rng = np.random.default_rng(1)
    D, H, P = 64, 2, 16
    k, v = rng.standard_normal((2, 37, H, D)) * np.exp(rng.standard_normal((2, 37, 1, 1)))
    table = np.array([[2, 0, 1]])
    made = []
    for pieces in ([37], [1] * 37, [5, 11, 1, 20]):
        c = ref.Cache(rng.integers(0, 256, (3, H, 1, 32 * D + 16)).astype(np.uint8), D, P)
        at = 0
        for n in pieces:
            c.append(k[at:at + n], k[at:at + n], v[at:at + n], table, [0, n], [at])
            at += n
        made.append(c.tokens(table, 0, 37)[0])
    for other in made[1:]:
        step = 2.0 ** np.ceil(np.log2(np.abs(made[0]).max() / 127))
        assert np.abs(other - made[0]).max() <= 1.5 * step
    assert np.abs(made[0][0] - k).max() <= np.abs(k).max() / 127  # half a step of the largest block's scale


def test_sampling_by_hand():
    x = np.log([4.0, 1, 3, 2])
    for u, want in ((0.0, 0), (0.39, 0), (0.41, 1), (0.51, 2), (0.79, 2), (0.81, 3), (0.999, 3)):
        assert ref.sample(x, u)[0] == want
    assert [ref.sample(x, u, k=2)[0] for u in (0.0, 0.56, 0.58, 0.99)] == [0, 0, 2, 2]
    assert [ref.sample(x, u, p=0.75)[0] for u in (0.44, 0.45, 0.99)] == [0, 2, 3]
    assert ref.sample(x, 0.99, p=0.69)[0] == 2 and ref.sample(x, 0.99, p=0.0)[0] == 0
    assert ref.sample(x, 0.99, m=0.6)[0] == 2 and ref.sample(x, 0.99, m=2.0)[0] == 0
    assert ref.sample(x, 0.99, T=0)[0] == 0 and ref.sample(np.full(4, -np.inf), 0.5)[0] == -1
    assert ref.sample(np.array([1.0, 1, 1]), 0.99, k=2)[0] == 1  # equal logits: by index


def test_kernels_wait_before_they_release():
    """A kernel's end implies that of all before it, and its operands may come from any call before it on the stream."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(tbuild.__file__), "csrc")
    for f, kernels in (("kv_append.cu", 2), ("kv_attend.cu", 1), ("sample.cu", 1)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, f)).read())
        assert len(re.findall(r"pdl_wait\(\);\s*pdl_release\(\);", text)) == kernels == text.count("pdl_release") == text.count("pdl_wait")


def test_no_cta_of_a_cluster_is_written_to_before_it_has_begun():
    """In the sampler's kernel a word is given at the start and awaited before anything that reaches another CTA."""
    import os
    import re
    text = re.sub(r"//[^\n]*", "", open(os.path.join(os.path.dirname(tbuild.__file__), "csrc", "sample.cu")).read())
    body = text[text.index("void run(const tetra_sample_rows& p"):]
    reaches = [m.start() for m in re.finditer(r"\bof\(|\btell\(|\bfind_bin<|\bgather\(|\bfind_cut<|\bsync\(\)", body)]
    assert body.count(" begun();") == body.count(" all_begun();") == 1 and reaches
    assert body.index(" begun();") < body.index("pdl_wait()") < body.index(" all_begun();") < min(reaches)
    assert "return" not in body[:body.index(" all_begun();")]
