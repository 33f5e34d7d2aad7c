"""The cache, its attention and the sampler between the products of a decode step, as a program runs them: embedding rows,
projections, append, attention, output projection, head, next token, which is the next step's input."""
import numpy as np
import pytest
import torch

import step_reference as ref
from paper_2609_35465_b200 import synth

pytestmark = pytest.mark.gpu

SEQS, HEADS, KV, D, HIDDEN, VOCAB, PAGE, WIDTH = 3, 8, 2, 128, 256, 5003, 32, 3
INV = 1e6 ** (-np.arange(0, D, 2) / D)


class Model:
    """One layer's attention and the head; the q projection is a Tetra matrix, the others are 4-bit."""

    def __init__(self, tt, seed=50):
        self.tt, self.table = tt, tt.tetra_build_table(synth.DEFAULT_GAIN)
        B = -(-HIDDEN // 24)
        self.q_codes = tt.tetra_pack_codes(torch.from_numpy(synth.codes(seed, 1, HEADS * D, B)).cuda().reshape(HEADS * D, B, 6), self.table, HEADS * D, B)
        self.q_scales = torch.from_numpy(synth.row_scales(seed, 1, HEADS * D)).cuda()
        self.mats = {}
        for i, (name, N, K, G) in enumerate((("k", KV * D, HIDDEN, 128), ("v", KV * D, HIDDEN, 128), ("o", HIDDEN, HEADS * D, 128), ("head", VOCAB, HIDDEN, 64))):
            s, o = synth.q4_scales_offsets(seed, i + 2, N, K // G)
            self.mats[name] = (tt.tetra_q4_pack(torch.from_numpy(synth.q4_nibbles(seed, i + 2, N, K)).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(o).cuda(), N, K, G), N, K, G)
        half = lambda *n: torch.zeros(n, dtype=torch.float16, device="cuda")  # noqa: E731
        full = lambda *n: torch.zeros(n, device="cuda")  # noqa: E731
        whole = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        g = torch.Generator("cuda").manual_seed(seed)
        self.cache = tt.tetra_kv_cache(SEQS * WIDTH + 1, PAGE, KV, D)
        self.cache.random_(generator=g)
        self.pages = whole(np.random.default_rng(seed).permutation(SEQS * WIDTH + 1)[:SEQS * WIDTH].reshape(SEQS, WIDTH))
        self.starts, self.lengths, self.tokens = whole(range(SEQS + 1)), whole([0, 0, 0]), whole([5, 77, 4999])
        self.x, self.qkv, self.q, self.att = half(SEQS, HIDDEN), full(3, SEQS, HEADS * D), half(SEQS, HEADS, D), half(SEQS, HEADS, D)
        self.k, self.v, self.y, self.logits = full(SEQS, KV * D), full(SEQS, KV * D), full(SEQS, HIDDEN), full(SEQS, VOCAB)
        self.weights = [1 + 0.1 * torch.randn(D, device="cuda", generator=g) for _ in range(2)]
        self.inv, self.ws, self.u, self.prob = torch.from_numpy(INV).cuda(), tt.tetra_kv_workspace(D), full(SEQS), full(SEQS)
        self.bws = torch.empty(tt.tetra_batched_workspace_bytes(HEADS * D, HIDDEN), dtype=torch.uint8, device="cuda")
        self.settings = dict(temperature=torch.tensor([0.7, 1.0, 0.0], device="cuda"), top_k=whole([20, 0, 0]), top_p=torch.tensor([0.9, 0.95, 1.0], device="cuda"))

    def q4(self, name, x, y):
        p, N, K, G = self.mats[name]
        self.tt.tetra_q4_gemv(p, x, y, N, K, G, SEQS)

    def step(self):
        tt, (head, N, K, G) = self.tt, self.mats["head"]
        cache = (self.cache, self.pages, self.starts, self.lengths)
        q = self.qkv[0]
        tt.tetra_q4_rows(head, self.tokens, self.x, N, K, G)
        tt.tetra_gemv_batched(self.q_codes, self.q_scales, self.table, self.x, q, HEADS * D, HIDDEN, SEQS, None, self.bws)
        self.q4("k", self.x, self.k)
        self.q4("v", self.x, self.v)
        tt.tetra_kv_append(q.view(SEQS, HEADS, D), self.k.view(SEQS, KV, D), self.v.view(SEQS, KV, D), *cache, self.q, inv_freq=self.inv, q_weight=self.weights[0], k_weight=self.weights[1])
        tt.tetra_kv_attend(self.q, *cache, self.att, self.ws)
        self.q4("o", self.att.view(SEQS, HEADS * D), self.y)
        self.x.add_(self.y)
        self.q4("head", self.x, self.logits)
        tt.tetra_sample(self.logits, self.u, self.tokens, prob=self.prob, **self.settings)
        self.lengths.add_(1)


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def test_steps_of_a_decode_loop(tt):
    """40 steps, over blocks and pages; each stage against its plain form on what the stage before made."""
    m, rng = Model(tt), np.random.default_rng(51)
    table, starts = m.pages.cpu().numpy(), np.arange(SEQS + 1)
    w = [x.cpu().numpy() for x in m.weights]
    for i in range(40):
        before = ref.Cache(m.cache.cpu().numpy(), D, PAGE)
        u = rng.random(SEQS).astype(np.float32)
        m.u.copy_(torch.from_numpy(u))
        m.step()
        n = [i] * SEQS
        q, k, v = (t.cpu().numpy().reshape(SEQS, -1, D) for t in (m.qkv[0], m.k, m.v))
        want = before.append(q, k, v, table, starts, n, INV, w[0], w[1], 1e-6)
        have = m.q.cpu().numpy()
        assert (np.abs(have - want) <= (2.0 ** -11 + 2.0 ** -40) * np.abs(want) + 2.0 ** -25).all()
        codes, scales = ref.unpack(m.cache.cpu().numpy(), D)
        for s in range(SEQS):
            page, block, t = before.place(table, s, i)
            assert np.array_equal(scales[page, :, block], before.scales[page, :, block])
            assert np.array_equal(codes[:, page, :, block, :t + 1], before.codes[:, page, :, block, :t + 1])
        o, bound = ref.attend(before, have, table, starts, n, 1 / np.sqrt(D))
        assert (np.abs(m.att.cpu().numpy() - o) <= bound).all()
        x, tokens = m.logits.cpu().numpy(), m.tokens.cpu().numpy()
        for s, (T, top_k, p) in enumerate(((0.7, 20, 0.9), (1.0, 0, 0.95), (0.0, 0, 1.0))):
            token, prob, far = ref.sample(x[s], u[s], float(np.float32(T)), top_k, float(np.float32(p)))
            assert far > VOCAB * 2.0 ** -44 and tokens[s] == token
            assert abs(float(m.prob[s]) - prob) <= 2.0 ** -24 * prob + VOCAB * 2.0 ** -43
    assert len({int(t) for t in m.tokens}) > 1


def test_a_captured_decode_loop(tt):
    """The whole step in one graph, its token fed back on the device, gives the tokens and the cache of the eager loop."""
    eager, graphed = Model(tt), Model(tt)
    graphed.cache.copy_(eager.cache)
    u = torch.rand((50, SEQS), device="cuda", generator=torch.Generator("cuda").manual_seed(52))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        graphed.step()
    seen = [[], []]
    for i in range(50):
        for out, m, run in ((seen[0], eager, eager.step), (seen[1], graphed, graph.replay)):
            m.u.copy_(u[i])
            run()
            out.append(m.tokens.clone())
    assert torch.equal(torch.stack(seen[0]), torch.stack(seen[1]))
    assert torch.equal(eager.cache, graphed.cache) and torch.equal(eager.prob, graphed.prob)
    assert not graphed.ws[:4608].any()


def test_first_calls_of_several_threads(tmp_path):
    """Four host threads, each with a stream and a workspace of its own, make the process's first calls at once."""
    import subprocess
    import sys
    program = tmp_path / "first.py"
    program.write_text("""
import threading
import torch
from paper_2609_35465_b200 import tetra
tetra._native()
torch.zeros(1, device="cuda")
gate, got, failed = threading.Barrier(4), [None] * 4, []

def work(i):
    try:
        torch.manual_seed(7)
        g = torch.Generator("cuda").manual_seed(7)
        with torch.cuda.stream(torch.cuda.Stream()):
            whole = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
            where = (tetra.tetra_kv_cache(8, 64, 2, 128), whole([[3, 1, 6, 0]]), whole([0, 250]), whole([0]))
            x = torch.randn((250, 12, 128), device="cuda", generator=g)
            q, out = torch.empty((2, 250, 8, 128), dtype=torch.float16, device="cuda")
            ws, logits, u, tokens = tetra.tetra_kv_workspace(128), torch.randn((5, 20000), device="cuda", generator=g), torch.rand(5, device="cuda", generator=g), whole([0] * 5)
            torch.cuda.current_stream().synchronize()
            gate.wait()
            tetra.tetra_kv_append(x[:, :8], x[:, 8:10], x[:, 10:], *where, q)
            tetra.tetra_kv_attend(q, *where, out, ws)
            tetra.tetra_sample(logits, u, tokens)
            torch.cuda.current_stream().synchronize()
            got[i] = out.cpu(), tokens.cpu()
    except Exception as e:
        failed.append(repr(e))
        gate.abort()

threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
for t in threads:
    t.start()
for t in threads:
    t.join()
assert not failed, failed
for o, t in got[1:]:
    assert torch.equal(o, got[0][0]) and torch.equal(t, got[0][1])
print("equal")
""")
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, str(program)], cwd=root, env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "equal" in run.stdout, run.stdout + run.stderr
