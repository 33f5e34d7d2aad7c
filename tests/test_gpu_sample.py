"""The choice of the next token on the GPU against the plain form in 64 bits (step_reference.sample).

The kernel's weights are whole multiples of 2^-44 that are off by no more than that, so every partial sum of n of them is off
by n 2^-44 in units of the largest weight; a draw whose aim is nearer to a border than that may fall on either
side, and none of those tested is (their distance is looked at).  prob is rounded to float32 once."""
import numpy as np
import pytest
import torch

import step_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def head_logits(rng, rows, vocab, dtype=np.float32):
    x = 2.5 * rng.standard_normal((rows, vocab))
    for r in range(rows):
        at = rng.integers(0, vocab, 24)
        x[r, at] += 6 + 7 * rng.random(24)
    return x.astype(dtype)


def check(tt, x, u, T=None, k=None, p=None, m=None, stride=None):
    rows, vocab = x.shape
    u = np.asarray(u, np.float32)
    d = torch.full((rows, stride or vocab), float("nan"), dtype=torch.float16 if x.dtype == np.float16 else torch.float32, device="cuda")
    d[:, :vocab] = torch.from_numpy(x)
    arr = lambda v, t: None if v is None else torch.tensor(np.broadcast_to(v, rows).copy(), dtype=t, device="cuda")  # noqa: E731
    tokens, prob = torch.full((rows,), -9, dtype=torch.int32, device="cuda"), torch.full((rows,), -9.0, device="cuda")
    args = dict(temperature=arr(T, torch.float32), top_k=arr(k, torch.int32), top_p=arr(p, torch.float32), min_p=arr(m, torch.float32))
    got = tt.tetra_sample(d[:, :vocab], torch.from_numpy(u).cuda(), tokens, prob=prob, **args)
    assert got is tokens
    again = torch.empty_like(tokens)
    tt.tetra_sample(d[:, :vocab], torch.from_numpy(u).cuda(), again, **args)
    assert torch.equal(tokens, again)
    at = lambda v, r, off: off if v is None else float(np.float32(np.broadcast_to(v, rows)[r]))  # noqa: E731
    for r in range(rows):
        token, q, far = ref.sample(x[r], u[r], at(T, r, 1.0), int(at(k, r, 0)), at(p, r, 1.0), at(m, r, 0.0))
        assert far > vocab * 2.0 ** -44, "the input lies next to a border"
        assert int(tokens[r]) == token, (r, int(tokens[r]), token)
        assert abs(float(prob[r]) - q) <= 2.0 ** -24 * q + vocab * 2.0 ** -43, (r, float(prob[r]), q)


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 1000, 4097, 32003, 151936])
def test_settings(tt, vocab, dtype):
    rng = np.random.default_rng(vocab)
    for T, k, p, m in ((None, None, None, None), (0.7, 20, 0.8, None), (1.3, None, 0.95, None), (1.0, 50, None, 0.05), (0.5, None, None, 0.01), (1.0, 1000, 0.999, None),
                       (2.0, 1, None, None), (0.9, None, 0.3, 0.2), (5.0, 4000, 0.99, None)):
        x = head_logits(rng, 3, vocab, dtype)
        check(tt, x, rng.random(3), T, k, p, m, stride=vocab + 5)


def test_rows_with_settings_of_their_own(tt):
    rng = np.random.default_rng(1)
    n = 40
    check(tt, head_logits(rng, n, 20011), rng.random(n), np.where(rng.random(n) < 0.2, 0, 0.3 + rng.random(n)), rng.integers(-1, 60, n),
          np.where(rng.random(n) < 0.3, 1.0, rng.random(n)), np.where(rng.random(n) < 0.5, 0, 0.1 * rng.random(n)))


@pytest.mark.parametrize("rows,vocab", [(2, 8191), (2, 8192), (2, 8193), (40, 32767), (40, 32768), (40, 32769), (90, 8200)])
def test_where_one_cta_takes_a_row(tt, rows, vocab):
    rng = np.random.default_rng(vocab)
    x = head_logits(rng, rows, vocab)
    for k, p, m in ((40, 0.9, None), (None, 0.9, None), (None, None, 0.001), (700, 0.97, None)):
        check(tt, x, rng.random(rows), 1.1, k, p, m)
    check(tt, np.zeros((rows, vocab), np.float32), rng.random(rows), 1.0, vocab // 2, 0.3)


@pytest.mark.parametrize("rows,vocab", [(14, 33000), (16, 33000), (21, 33001), (24, 33003), (30, 33000), (33, 40000), (45, 33000), (20, 262144), (18, 350001)])
def test_clusters_of_every_size(tt, rows, vocab):
    """Numbers of rows for which clusters of eight, six, five, four and again eight CTAs are taken, and rows too long for the smaller ones."""
    rng = np.random.default_rng(rows)
    x = head_logits(rng, rows, vocab)
    for k, p, m in ((40, 0.9, None), (128, None, 0.01), (None, 0.9, None), (None, None, 0.001), (700, 0.97, None)):
        check(tt, x, rng.random(rows), 1.1, k, p, m)
    few = np.full((rows, vocab), -np.inf, np.float32)
    few[:, rng.integers(0, vocab, 40)] = 3 * rng.standard_normal((rows, 40))
    check(tt, few, rng.random(rows), 2.0, 60, 0.95)
    if vocab < 50000:  # more equal logits than a part's share of the list
        check(tt, np.zeros((rows, vocab), np.float32), rng.random(rows), 1.0, 100, 0.3)
        check(tt, np.zeros((rows, vocab), np.float32), rng.random(rows), 1.0, None, 0.3)


def test_largest_vocabulary(tt):
    rng = np.random.default_rng(2)
    check(tt, head_logits(rng, 2, 393216), rng.random(2), 1.0, None, 0.9)


def test_equal_logits_go_by_index(tt):
    """One value for all, two values, whole numbers: bins with more entries than are sorted, cut inside equal ones."""
    rng = np.random.default_rng(3)
    u = [0.05, 0.51, 0.97]
    for vocab in (3, 100, 5000, 70001):
        for x in (np.zeros((3, vocab)), np.full((3, vocab), -7.25), (np.arange(3 * vocab) % 2).reshape(3, vocab) * 1.0, rng.integers(0, 4, (3, vocab)) * 1.0):
            x = x.astype(np.float32)
            for k, p in ((None, None), (max(1, vocab // 3), None), (None, 0.37), (vocab, 0.5), (max(1, vocab - 1), 0.73)):
                check(tt, x, u, 1.0, k, p)


def test_zeros_of_either_sign_are_equal(tt):
    x = np.array([[-0.0, 0.0, -0.0, -1]] * 3, np.float32)
    check(tt, x, [0.2, 0.6, 0.95], 1.0, 2)
    check(tt, x, [0.2, 0.6, 0.95], 0.0)


def test_outliers_and_masks(tt):
    """The type's lowest value and minus infinity as masks, one logit far above or below the others."""
    rng = np.random.default_rng(4)
    for low in (-np.inf, np.finfo(np.float32).min, -65504.0, -1e9):
        x = head_logits(rng, 4, 30011)
        x[rng.random(x.shape) < 0.7] = low
        check(tt, x, rng.random(4), 1.0, 2000, 0.97)
        check(tt, x, rng.random(4), 1.0)
    for T in (0.1, 1.0, 300.0):
        x = head_logits(rng, 4, 30011)
        x[:, 17] = 1000
        x[2:, 99] = -1e30
        check(tt, x, rng.random(4), T, 5000, 0.98)
    x = np.full((2, 1000), np.finfo(np.float32).min, np.float32)
    check(tt, x, [0.3, 0.7], 1.0, 10, 0.9)
    x[:, 5] = np.finfo(np.float32).max
    check(tt, x, [0.3, 0.7], 1.0, 10, 0.9)
    check(tt, x, [0.3, 0.7], 1e38, 10, 0.9)


@pytest.mark.parametrize("vocab,last", [(40, 39), (9001, 9000), (9001, 39), (151936, 151935), (151936, 39)])
def test_fewer_tokens_than_top_k(tt, vocab, last):
    """Two or three logits above minus infinity, of any fractions: the least, whose distance from the largest is not a float32,
    has its mass too."""
    rng = np.random.default_rng(5)
    n = 24
    x = np.full((n, vocab), -np.inf, np.float32)
    x[:, 3] = 8 + 8 * rng.random(n)
    x[:, last] = rng.random(n)
    x[::2, 20] = 4 + rng.random(n // 2)
    check(tt, x, np.full(n, 0.999), 8.0, 30)
    check(tt, x, np.full(n, 0.999), 8.0, 30, None, 0.01)


def test_flat_distributions(tt):
    """High temperatures and small logits: everything lies within a few bins of the largest."""
    rng = np.random.default_rng(5)
    x = (0.01 * rng.standard_normal((3, 50021))).astype(np.float32)
    check(tt, x, rng.random(3), 1.0, 20000, 0.5)
    check(tt, head_logits(rng, 3, 50021), rng.random(3), 1000.0, None, 0.7)
    check(tt, head_logits(rng, 3, 50021), rng.random(3), np.inf, 100, 0.7)


def test_rows_without_a_token_and_what_is_not_finite(tt):
    x = np.full((6, 500), -np.inf, np.float32)
    x[1] = np.nan
    x[2, 400] = -3.0
    x[3, [7, 300, 301]] = np.inf
    x[4] = np.linspace(-5, 5, 500)
    x[4, ::2] = np.nan
    x[5] = np.linspace(-5, 5, 500)
    x[5, 100] = np.inf
    for T in (1.0, 0.0):
        for k, p, m in ((None, None, None), (2, 0.9, 0.1)):
            check(tt, x, [0.5, 0.5, 0.5, 0.6, 0.3, 0.3], T, k, p, m)


def test_ends_of_u_and_odd_settings(tt):
    rng = np.random.default_rng(6)
    x = head_logits(rng, 8, 999)
    tokens = torch.zeros(8, dtype=torch.int32, device="cuda")
    u = torch.tensor([0.0, 1.0, -3.0, 7.0, float("nan"), float("inf"), -float("inf"), 1 - 2.0 ** -24], device="cuda")
    tt.tetra_sample(torch.from_numpy(x).cuda(), u, tokens, top_k=torch.full((8,), 5, dtype=torch.int32, device="cuda"))
    for r in range(8):
        kept = np.sort(np.argsort(-x[r], kind="stable")[:5])
        assert int(tokens[r]) == (kept[0] if r in (0, 2, 4, 6) else kept[-1])
    # p of zero or below, or m above one: the first alone; p of NaN, m and k below zero: off
    check(tt, x, rng.random(8), 1.0, [0, -5, 0, 0, 2, 0, 3, 0], [0.0, -1.0, 1.0, 2.0, 1.0, 1e-30, 1.0, 1.0], [0.0, 0.0, 2.0, -1.0, 0.0, 0.0, 1.0, np.inf])
    check(tt, x, rng.random(8), [-1.0, 0.0, np.nan, 1e-30, 1e30, 1.0, 1.0, 1.0])
    want, got = torch.empty_like(tokens), torch.empty_like(tokens)
    d, r8 = torch.from_numpy(x).cuda(), torch.rand(8, device="cuda")
    tt.tetra_sample(d, r8, want)
    tt.tetra_sample(d, r8, got, top_p=torch.full((8,), float("nan"), device="cuda"), min_p=torch.full((8,), float("nan"), device="cuda"))
    assert torch.equal(want, got)


def test_draws_follow_the_distribution(tt):
    """4096 even values of u: each token as often as its mass says, but for one at either end."""
    n = 4096
    x = np.log(np.array([8.0, 1, 4, 2, 1, 16]))
    d = torch.from_numpy(np.tile(x, (n, 1)).astype(np.float32)).cuda()
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tokens = torch.empty(n, dtype=torch.int32, device="cuda")
    tt.tetra_sample(d, u, tokens, top_k=torch.full((n,), 4, dtype=torch.int32, device="cuda"))
    have = torch.bincount(tokens, minlength=6).cpu().numpy()
    assert (np.abs(have - n * np.array([8, 0, 4, 2, 0, 16]) / 30) <= 1).all()


def test_captured_and_on_another_stream(tt):
    rng = np.random.default_rng(7)
    x = torch.from_numpy(head_logits(rng, 5, 10007)).cuda()
    u, tokens = torch.rand(5, device="cuda"), torch.empty(5, dtype=torch.int32, device="cuda")
    p = torch.full((5,), 0.9, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tt.tetra_sample(x, u, tokens, top_p=p)
    for _ in range(5):
        u.copy_(torch.rand(5, device="cuda"))
        x.copy_(torch.from_numpy(head_logits(rng, 5, 10007)))
        graph.replay()
        want = tt.tetra_sample(x, u, torch.empty_like(tokens), top_p=p)
        assert torch.equal(tokens, want)
    torch.cuda.synchronize()
    other = torch.empty_like(tokens)
    tt.tetra_sample(x, u, other, top_p=p, stream=side)
    side.synchronize()
    assert torch.equal(tokens, other)


def test_the_binding_refuses(tt):
    x, u, t = torch.zeros((2, 10), device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def refused(match, *args, **more):
        with pytest.raises(tt.TetraError, match=match):
            tt.tetra_sample(*args, **more)
    refused("logits: BFloat16", x.bfloat16(), u, t)
    refused("logits: wrong shape", x[0], u, t)
    refused("logits: wrong shape", x.t().contiguous().t(), u, t)
    refused("u: Double", x, u.double(), t)
    refused("u: wrong", x, u[:1], t)
    refused("tokens: Long", x, u, t.long())
    refused("tokens: tensor is not on the device", x, u, t.cpu())
    refused("temperature: wrong", x, u, t, temperature=u[:1])
    refused("top_k: Float", x, u, t, top_k=u)
    refused("top_p: tensor is not contiguous", x, u, t, top_p=torch.zeros(4, device="cuda")[::2])
    refused("prob: wrong", x, u, t, prob=u[:1])
    refused("out of range", x[:1].expand(2, 10), u, t)
    refused("out of range", torch.zeros((1, 393217), device="cuda"), u[:1], t[:1])
    refused("out of range", torch.zeros((2, 0), device="cuda"), u, t)
    assert tt.tetra_sample(x[:0], u[:0], t[:0]) is not None
