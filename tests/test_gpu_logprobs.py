"""Log probabilities, ranks, entropy and likeliest tokens on the GPU against the plain form in 64 bits.

Whole numbers are equal.  A logarithm of a sum of n weights is off by the sum's relative error: a weight 2^z by 2^-22 (the instruction) and
by |z| ln 2 2^-22 (its argument's three roundings), which the weights' mean of |z|, ln(n) / ln 2 at most, counts; float32 additions
of 16 terms, of a thread's tiles and of four more by 2^-24 each.  For n <= 400000 that is below 2^-22 (1 + 13) + 2^-24 (16 + 50 + 4)
< 2^-17; the result is rounded once, 2^-24 of itself.  The entropy is that plus the mean of -z, off by as much of itself."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LARGEST = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def plain(x, tokens, T, top):
    """(logprob, rank, entropy, top tokens, top logprob) of one row; float64."""
    x = np.asarray(x).astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, np.where(x == np.inf, LARGEST, np.where(np.abs(x) < 2.0 ** -126, 0, x)))
    order = np.argsort(-x, kind="stable")
    place = np.empty(x.size, np.int64)
    place[order] = np.arange(x.size)
    most = x[order[0]]
    if most == -np.inf:
        lp, entropy = np.full(x.size, -np.inf), 0.0
    elif not T > 0:
        lp, entropy = np.full(x.size, -np.inf), 0.0
        lp[order[0]] = 0
    else:
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            z = np.where(x == -np.inf, -np.inf, (x - most) / T)
            e = np.exp(z)
            lp = z - np.log(e.sum())
            p = e / e.sum()
            entropy = -(p[p > 0] * lp[p > 0]).sum()
    given = [(lp[t], place[t]) if 0 <= t < x.size else (-np.inf, -1) for t in tokens]
    first = [t if x[t] > -np.inf else -1 for t in order[:top]]
    first += [-1] * (top - len(first))
    return [g[0] for g in given], [g[1] for g in given], entropy, first, [lp[t] if t >= 0 else -np.inf for t in first]


def near(have, want, what):
    have, want = np.asarray(have, np.float64), np.asarray(want, np.float64)
    want = np.where(want < -LARGEST, -np.inf, want)
    assert not np.isnan(have).any(), what
    same = have == want
    with np.errstate(invalid="ignore"):
        off = np.abs(have - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -17
    assert (same | off).all(), (what, have[~(same | off)][:4], want[~(same | off)][:4])


def check(tt, x, tokens=None, T=None, top=0, rows_of=None):
    """x: a device tensor [rows, vocab]; tokens: array [rows, given]."""
    R, V = x.shape
    given = 0 if tokens is None else tokens.shape[1]
    i = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *s: torch.full(s, 7.5, device="cuda")  # noqa: E731
    t = None if tokens is None else torch.tensor(tokens, dtype=torch.int32, device="cuda")
    lp, rank, entropy, tops, top_lp = f(R, given) if given else None, i(R, given) if given else None, f(R), i(R, top) if top else None, f(R, top) if top else None
    d_T = None if T is None else torch.tensor(np.asarray(T), dtype=torch.float32, device="cuda")
    call = lambda: tt.tetra_logprobs(x, t, lp, rank=rank, entropy=entropy, top_tokens=tops, top_logprob=top_lp, temperature=d_T)  # noqa: E731
    assert call() is lp
    outs = [o.cpu().numpy().copy() for o in (lp, rank, entropy, tops, top_lp) if o is not None]
    call()
    for a, b in zip(outs, [o.cpu().numpy() for o in (lp, rank, entropy, tops, top_lp) if o is not None]):
        assert np.array_equal(a.view(np.int32), b.view(np.int32))
    host = x.float().cpu().numpy()
    for r in (range(R) if rows_of is None else rows_of):
        temp = 1.0 if T is None else float(np.float32(T[r]))
        want = plain(host[r], [] if tokens is None else tokens[r], temp, top)
        if given:
            assert rank[r].tolist() == list(want[1]), (r, rank[r].tolist(), want[1])
            near(lp[r].cpu().numpy(), want[0], ("logprob", r))
        have = float(entropy[r])
        assert abs(have - want[2]) <= 2.0 ** -24 * abs(want[2]) + 2.0 ** -17 * (1 + abs(want[2])), ("entropy", r, have, want[2])
        if top:
            assert tops[r].tolist() == [int(v) for v in want[3]], r
            near(top_lp[r].cpu().numpy(), want[4], ("top", r))


def logits(seed, R, V, dtype=torch.float32):
    g = torch.Generator("cuda").manual_seed(seed)
    x = 2.5 * torch.randn((R, V), device="cuda", generator=g)
    at = torch.randint(0, V, (R, 5), device="cuda", generator=g)
    return x.scatter_add_(1, at, 8 * torch.rand((R, 5), device="cuda", generator=g)).to(dtype)


def some(seed, R, V, n):
    return np.random.default_rng(seed).integers(0, V, (R, n))


# Sizes about those at which tiles, clusters and kernels change.
@pytest.mark.parametrize("V", [1, 2, 3, 7, 33, 127, 128, 1000, 2047, 2048, 2049, 8191, 8192, 8193, 16387, 32003, 65535, 65537, 151936, 262147])
@pytest.mark.parametrize("R,dtype,given,top", [(1, torch.float32, 1, 5), (3, torch.float16, 4, 20), (19, torch.float32, 1, 1)])
def test_sizes(tt, V, R, dtype, given, top):
    check(tt, logits(V + R, R, V, dtype), some(V, R, V, given), top=top)


@pytest.mark.parametrize("R,V", [(1, 40000), (18, 70001), (19, 70001), (74, 9001), (75, 9001), (83, 9001), (84, 9001), (148, 8200), (150, 8200), (166, 8200), (170, 8200), (333, 8200), (340, 8200), (700, 9000), (1500, 700), (65535, 5)])
def test_numbers_of_rows(tt, R, V):
    check(tt, logits(R, R, V), some(R, R, V, 2), top=3, rows_of=sorted({0, 1, R // 2, R - 1} & set(range(R))))


@pytest.mark.parametrize("R", [15, 16, 36, 37, 74, 75, 148, 149])
@pytest.mark.parametrize("V,dtype,top", [(16385, torch.float16, 20), (40003, torch.float32, 32), (140001, torch.float32, 16)])
def test_numbers_of_long_rows(tt, R, V, dtype, top):
    check(tt, logits(R + V, R, V, dtype), some(R, R, V, 1), top=top, rows_of=[0, R // 2, R - 1])


@pytest.mark.parametrize("given,top", [(0, 0), (0, 32), (64, 0), (64, 32), (5, 8), (2, 9), (1, 31)])
@pytest.mark.parametrize("R,V", [(2, 5003), (2, 100003), (40, 20011), (200, 9001)])
def test_numbers_of_tokens(tt, R, V, given, top):
    tokens = some(R, R, V, given) if given else None
    if given > 1:
        tokens[:, 1] = tokens[:, 0]  # twice the same
    check(tt, logits(7, R, V, torch.float16 if top % 2 else torch.float32), tokens, top=top, rows_of=[0, R - 1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("V", [1003, 9001, 70001])
def test_rows_that_lie_apart_at_odd_places(tt, V, dtype):
    wide = logits(11, 9, V + 13, dtype)
    for offset in range(9):
        check(tt, wide[:, offset:offset + V], some(offset, 9, V, 1), top=4, rows_of=[0, 3, 8])


@pytest.mark.parametrize("V", [100, 4001, 33000, 151936])
def test_equal_logits(tt, V):
    x = torch.zeros((4, V), device="cuda")
    x[1] = torch.arange(V, device="cuda") % 3
    x[2] = -(torch.arange(V, device="cuda") % 7).float() / 3
    x[3, V // 2:] = -0.0
    tokens = np.array([[0, V - 1, V // 2, 1]] * 4)
    check(tt, x, tokens, top=32)
    check(tt, x.half(), tokens, top=7)


@pytest.mark.parametrize("V", [500, 8192, 8193, 60000, 151936, 400000])
@pytest.mark.parametrize("top", [1, 8, 9, 32])
def test_rising_and_falling_logits(tt, V, top):
    """Every logit is the largest so far: there are more candidates than any list has room for."""
    up = torch.arange(V, device="cuda") * 2.0 ** -12
    x = torch.stack([up, up.flip(0), torch.where(torch.arange(V, device="cuda") < V // 2, up, up.flip(0)), up % 1])
    check(tt, x, some(3, 4, V, 2), top=top)
    if V > 60000:
        check(tt, x.repeat(200, 1), None, top=top, rows_of=[0, 1, 398, 799])


@pytest.mark.parametrize("V", [50, 5003, 40000, 151936])
def test_what_is_not_a_number(tt, V):
    g = np.random.default_rng(V)
    x = logits(13, 12, V).cpu().numpy()
    x[0, g.random(V) < 0.5] = -np.inf
    x[1] = -np.inf
    x[2] = np.nan
    x[3, g.random(V) < 0.3] = np.nan
    x[4, V // 3], x[4, V // 2] = np.inf, np.inf
    x[5, V // 3], x[5, V // 2] = np.inf, LARGEST
    x[6] = -np.inf
    x[6, V - 1] = -5
    x[7] = LARGEST
    x[8] = -LARGEST
    x[9] *= 2.0 ** -130                    # zeros, all of them
    x[10, :V // 2], x[10, V // 2:] = 3e38, -3e38
    x[11] = np.inf
    tokens = np.concatenate([some(1, 12, V, 3), np.tile([V // 3, V // 2, 0, V - 1, -1, V, 2 ** 31 - 1, -2 ** 31], (12, 1))], 1)
    check(tt, torch.from_numpy(x).cuda(), tokens, top=6)


@pytest.mark.parametrize("V", [300, 20000, 151936])
def test_temperatures(tt, V):
    T = [1.0, 0.5, 2.0, 0.0, -1.0, np.nan, np.inf, 1e-30, 1e30, 1e-3, 1e-45, 100.0]
    x = logits(17, len(T), V)
    x[3, [V - 1, 5]] = 50.0  # of equal largest ones the first
    check(tt, x, np.concatenate([some(5, len(T), V, 2), np.tile([5, V - 1], (len(T), 1))], 1), T=T, top=5)
    x[:] = -np.inf
    check(tt, x, some(5, len(T), V, 1), T=T, top=2)


def test_a_distribution_on_one_token(tt):
    """Probabilities next to 1: the log probability is minus the others' mass, absolutely as near as stated."""
    x = torch.full((2, 50000), -20.0, device="cuda")
    x[:, 777] = torch.tensor([10.0, 40.0], device="cuda")
    check(tt, x, np.array([[777, 3]] * 2), top=2)


def test_offsets_that_pass_32_bits(tt):
    V, R = 300000, 8000
    x = torch.empty((R, V), dtype=torch.float16, device="cuda").normal_()
    assert x.numel() * 2 > 2 ** 32
    check(tt, x, some(9, R, V, 1), top=3, rows_of=[0, 7159, 7999])


# ---- streams, graphs, refusals -----------------------------------------------------------------------------------------
def test_a_captured_call_follows_its_inputs(tt):
    for R, V in ((1, 151936), (40, 30000), (300, 2000)):
        x, t, T = torch.zeros((R, V), device="cuda"), torch.zeros((R, 2), dtype=torch.int32, device="cuda"), torch.ones(R, device="cuda")
        outs = lambda: (torch.zeros((R, 2), device="cuda"), dict(rank=torch.zeros((R, 2), dtype=torch.int32, device="cuda"), entropy=torch.zeros(R, device="cuda"),  # noqa: E731
                        top_tokens=torch.zeros((R, 4), dtype=torch.int32, device="cuda"), top_logprob=torch.zeros((R, 4), device="cuda")))
        lp, more = outs()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            tt.tetra_logprobs(x, t, lp, temperature=T, **more)
        for i in range(3):
            x.copy_(logits(i, R, V)), t.copy_(torch.tensor(some(i, R, V, 2))), T.uniform_(0.3, 2)
            graph.replay()
            lp2, more2 = outs()
            tt.tetra_logprobs(x, t, lp2, temperature=T, **more2)
            assert torch.equal(lp, lp2) and all(torch.equal(more[k], more2[k]) for k in more)


def test_two_streams(tt):
    x, t = logits(3, 5, 60000), torch.tensor(some(3, 5, 60000, 1), dtype=torch.int32, device="cuda")
    want = tt.tetra_logprobs(x, t, torch.empty((5, 1), device="cuda"))
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty((5, 1), device="cuda") for _ in range(40)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        tt.tetra_logprobs(x, t, o, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_the_binding_refuses(tt):
    x, t, lp = torch.zeros((2, 100), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")

    def refused(match, *args, **more):
        with pytest.raises(tt.TetraError, match=match):
            tt.tetra_logprobs(*args, **more)
    refused("logits: Double", x.double(), t, lp)
    refused("logits: wrong", x[0], t, lp)
    refused("logits: wrong", x.t(), t, lp)
    refused("tokens: Long", x, t.long(), lp)
    refused("tokens: wrong", x, t[:1], lp)
    refused("logprob: wrong", x, t, lp[:, :2].contiguous())
    refused("tokens and logprob", x, None, lp)
    refused("tokens and logprob", x, t, None)
    refused("rank is that of", x, None, None, rank=t)
    refused("rank: Float", x, t, lp, rank=lp)
    refused("entropy: wrong", x, t, lp, entropy=lp)
    refused("top_tokens and top", x, t, lp, top_tokens=t)
    refused("top_logprob: wrong", x, t, lp, top_tokens=t, top_logprob=lp[:, :2].contiguous())
    refused("temperature: wrong", x, t, lp, temperature=lp[0])
    refused("out of range", x, torch.zeros((2, 65), dtype=torch.int32, device="cuda"), torch.zeros((2, 65), device="cuda"))
    refused("out of range", x, t, lp, top_tokens=torch.zeros((2, 33), dtype=torch.int32, device="cuda"), top_logprob=torch.zeros((2, 33), device="cuda"))
    refused("out of range", x[:, :0], t, lp)
    refused("out of range", x[:1].expand(2, 100), t, lp)
    none = torch.zeros((0, 3), device="cuda")
    assert tt.tetra_logprobs(x[:0], t[:0], none) is none
    assert tt.tetra_logprobs(x, None, None, entropy=torch.zeros(2, device="cuda")) is None


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_the_longest_rows(tt, dtype):
    """2^24 logits: the sums' terms are 42 times those of 400000, added by 8192 threads; (50 + 3700 of a thread's tiles) 2^-24 is below 2^-12."""
    V = 1 << 24
    x = logits(31, 2, V, dtype)
    lp, top, top_lp, rank, entropy = (torch.empty(s, device="cuda", dtype=t) for s, t in (((2, 1), torch.float32), ((2, 8), torch.int32), ((2, 8), torch.float32), ((2, 1), torch.int32), ((2,), torch.float32)))
    t = torch.tensor([[V - 1], [5]], dtype=torch.int32, device="cuda")
    tt.tetra_logprobs(x, t, lp, rank=rank, entropy=entropy, top_tokens=top, top_logprob=top_lp)
    want = torch.log_softmax(x.double(), -1)
    assert (lp.double() - want.gather(1, t.long())).abs().max() <= 2.0 ** -12
    assert (entropy.double() + (want.exp() * want).sum(-1)).abs().max() <= 2.0 ** -8
    order = torch.sort(x.float(), dim=-1, descending=True, stable=True).indices
    assert torch.equal(top.long(), order[:, :8])
    assert torch.equal(rank.long()[:, 0], (order == t.long()).nonzero()[:, 1])
