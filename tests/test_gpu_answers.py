"""The operators as a server uses them together: a picture's rows go into the cache at positions of their own, several answers behind it
attend to what they share, and what was answered is scored.  Eager and as one graph; against the plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import step_reference as ref
from test_gpu_kv import INV, Step, dev, i32
from test_gpu_kv_append_at import plain_rows
from test_gpu_kv_shared import share
from test_gpu_logprobs import near, plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tt():
    from paper_2609_35465_b200 import tetra
    return tetra


def test_a_picture_its_answers_and_their_worth(tt):
    D, H, heads, P, V, top = 128, 2, 8, 16, 5003, 4
    high, wide, text, answers = 12, 15, 28, 5
    prompt = high * wide + text                                      # 208 tokens, which all answers share
    st = Step(401, D, H, P, [0] * answers, [1] * answers, width=20)
    start, shared = share(st, [(0, answers, prompt)])
    plain_cache = st.plain()
    rng = st.rng

    # The prompt: a picture (time, height, width), then text on all three axes.
    axis = np.repeat([0, 1, 2], [16, 24, 24]).astype(np.uint8)
    picture = np.stack(np.meshgrid([7], np.arange(high), np.arange(wide), indexing="ij"), -1).reshape(-1, 3) + [0, 7, 7]
    after = np.arange(text)[:, None] + [7 + max(high, wide)] * 3
    positions = np.concatenate([picture, after])
    x = rng.standard_normal((prompt, heads + 2 * H, D)).astype(np.float32)
    d_axis, inv = dev(axis), dev(INV[D])
    first = i32([0, prompt])
    one = i32(st.table[:1])
    zero = i32([0])

    # A step of the answers.
    y = rng.standard_normal((answers, heads + 2 * H, D)).astype(np.float32)
    lengths = np.full(answers, prompt)
    next_positions = np.tile(positions[-1] + 1, (answers, 1))
    logits = torch.from_numpy(rng.standard_normal((answers, V)).astype(np.float32) * 3).cuda()
    tokens = rng.integers(0, V, (answers, 1)).astype(np.int32)

    d_x, d_y, d_pos, d_next, d_tokens, d_lengths = dev(x), dev(y), i32(positions), i32(next_positions), dev(tokens), i32(list(lengths) + [0] * (len(st.d_lengths) - answers))
    half = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")  # noqa: E731
    q0, q1, out = half(prompt, heads, D), half(answers, heads, D), half(answers, heads, D)
    lp, rank = torch.zeros((answers, 1), device="cuda"), torch.zeros((answers, 1), dtype=torch.int32, device="cuda")
    tops, top_lp, entropy = torch.zeros((answers, top), dtype=torch.int32, device="cuda"), torch.zeros((answers, top), device="cuda"), torch.zeros(answers, device="cuda")
    ws = tt.tetra_kv_shared_workspace(D, answers, heads, H, 1)

    def run():
        tt.tetra_kv_append_at(d_x[:, :heads], d_x[:, heads:heads + H], d_x[:, heads + H:], st.cache, one, first, zero, d_pos, d_axis, q0, inv)
        tt.tetra_kv_append_at(d_y[:, :heads], d_y[:, heads:heads + H], d_y[:, heads + H:], st.cache, st.d_table, st.d_starts, d_lengths, d_next, d_axis, q1, inv)
        tt.tetra_kv_attend_shared(q1, st.cache, st.d_table, st.d_starts, d_lengths, start, shared, out, ws)
        tt.tetra_logprobs(logits, d_tokens, lp, rank=rank, entropy=entropy, top_tokens=tops, top_logprob=top_lp)
        return [t.clone() for t in (st.cache, q0, q1, out, lp, rank, entropy, tops, top_lp)]

    eager = run()
    st.cache.copy_(dev(st.raw))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        again = run()
    for _ in range(2):
        st.cache.copy_(dev(st.raw))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(eager, again))

    # The plain forms.
    turned = [plain_rows(x[:, a:b], None, positions, axis, INV[D]) for a, b in ((0, heads), (heads, heads + H))]
    plain_cache.append(turned[0], turned[1], x[:, heads + H:], st.table[:1], [0, prompt], [0])
    turned = [plain_rows(y[:, a:b], None, next_positions, axis, INV[D]) for a, b in ((0, heads), (heads, heads + H))]
    plain_cache.append(turned[0], turned[1], y[:, heads + H:], st.table, st.starts, lengths)
    want, bound = ref.attend(plain_cache, q1.cpu().numpy(), st.table, st.starts, lengths, 1 / np.sqrt(D))
    bound = bound * (2 + ((prompt + 1) / 16 + 64) * 2.0 ** -12)   # as for groups
    assert (np.abs(out.cpu().numpy() - want) <= bound).all()
    for r in range(answers):
        one_row = plain(logits[r].cpu().numpy(), tokens[r], 1.0, top)
        assert rank[r].tolist() == list(one_row[1]) and tops[r].tolist() == [int(t) for t in one_row[3]]
        near(lp[r].cpu().numpy(), one_row[0], r)
        near(top_lp[r].cpu().numpy(), one_row[4], r)
