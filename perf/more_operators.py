"""Operators for several answers behind one prompt, as cases that can be timed and compared: a prompt with pictures in it is
appended to the 8-bit paged cache, the answers' tokens attend to it together, and tokens are scored.

  append   rows at given positions of several axes (time, height, width) into the cache, and what they became read back:
           tetra_kv_append_at + tetra_kv_read
  attend   attention of groups of sequences whose first tokens are the same pages of the cache: tetra_kv_attend_shared
  score    log probabilities and ranks of given tokens, the entropy of their distribution and the likeliest tokens:
           tetra_logprobs

The cache is that of tetra_kv.h: for each page, kv head and block of 16 tokens a record of 32 D + 16 bytes, 16 D bytes of keys,
16 D of values (code + 128; the orders stand above `_codes_of`), two float32 scales that are powers of two, eight bytes without
meaning.  `row_start` says which rows belong to which sequence, `lengths` how many tokens each sequence had before these rows.

Shapes are those of shapes.py (dense models with 32 or 40 query heads and 8 kv heads of 128, a vocabulary of 151936) and
generic sizes around them.
"""
import math

import torch

own = False

DEVICE = "cuda"
BLOCK = 16


def listed():
    heads8, heads14 = dict(q_heads=32, kv_heads=8, dim=128), dict(q_heads=40, kv_heads=8, dim=128)
    return [
        # one token of one 8B sequence behind pictures (its position is not its slot): the step of a chat, latency is all there is
        dict(name="append_1_8b", op="append", seqs=1, chunk=1, grid=0, low=900, high=900, page=64, dtype="float32", norm=True, idle=False, **heads8),
        # a server's batch of the 14B model, ragged, one slot without a token, padded to a fixed batch
        dict(name="append_64_14b", op="append", seqs=64, chunk=1, grid=0, low=1, high=900, page=32, dtype="float32", norm=True, idle=True, **heads14),
        # a picture of 56 x 52 patches behind a question, odd beginning inside a block
        dict(name="append_picture_8b", op="append", seqs=1, chunk=56 * 52, grid=52, low=37, high=37, page=64, dtype="float32", norm=True, idle=False, **heads8),
        # two answers of one short prompt: the smallest call that has something to share
        dict(name="attend_2_on_320_8b", op="attend", groups=1, seqs=2, chunk=1, shared=320, low=1, high=40, page=64, alone=False, idle=False, **heads8),
        # sixteen answers of the 14B model (five query heads to a kv head), ragged, one slot without a sequence
        dict(name="attend_16_on_2048_14b", op="attend", groups=1, seqs=16, chunk=1, shared=2048, low=1, high=500, page=32, alone=False, idle=True, **heads14),
        # four prompts of different lengths, eight answers each, and a sequence that shares nothing
        dict(name="attend_4x8_ragged_8b", op="attend", groups=4, seqs=8, chunk=1, shared=6000, low=20, high=700, page=16, alone=True, idle=False, **heads8),
        # a question's choices, several tokens each, scored at once
        dict(name="attend_choices_8b", op="attend", groups=1, seqs=5, chunk=12, shared=1500, low=0, high=3, page=16, alone=False, idle=False, **heads8),
        # the largest batch: 64 answers behind one long document
        dict(name="attend_64_on_16384_8b", op="attend", groups=1, seqs=64, chunk=1, shared=16384, low=100, high=1024, page=128, alone=False, idle=False, **heads8),
        # the token that was just sampled, and five alternatives
        dict(name="score_1_head", op="score", rows=1, vocab=151936, dtype="float32", given=1, top=5, heated=False),
        # a small vocabulary of odd size in half precision (many equal logits), four choices each, temperatures of their own
        dict(name="score_7x32003", op="score", rows=7, vocab=32003, dtype="float16", given=4, top=20, heated=True),
        # a server's batch
        dict(name="score_64_head", op="score", rows=64, vocab=151936, dtype="float32", given=1, top=20, heated=False),
        # the tokens of a prompt
        dict(name="score_prompt_1024", op="score", rows=1024, vocab=151936, dtype="float32", given=1, top=1, heated=False),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "score", "attend"])
    if op == "score":
        vocab = _spread(rng, 500, 262144)
        return dict(op=op, rows=_spread(rng, 1, max(1, min(4000, 1024 * 151936 // vocab))), vocab=vocab, dtype=rng.choice(["float32", "float16"]),
                    given=rng.choice([1, 1, rng.randint(2, 8)]), top=rng.choice([0, 1, 5, rng.randint(2, 32)]), heated=rng.random() < 0.4)
    q_heads, kv_heads = rng.choice([(32, 8), (40, 8), (16, 2), (8, 8), (7, 1), (24, 2)])
    case = dict(op=op, q_heads=q_heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128, 128, 256]), page=rng.choice([16, 32, 48, 64, 128]), idle=rng.random() < 0.3)
    if op == "append":
        chunk = rng.choice([1, rng.randint(2, 16), _spread(rng, 17, 2900)])
        seqs = _spread(rng, 1, max(1, min(64, 2900 // chunk)))
        high = _spread(rng, 1, 1000)
        case.update(seqs=seqs, chunk=chunk, grid=rng.choice([0, rng.randint(1, 64)]), low=rng.randint(0, high), high=high,
                    dtype=rng.choice(["float32", "float16"]), norm=rng.random() < 0.5, idle=case["idle"] and seqs > 1)
        size = chunk * seqs * (q_heads + 2 * kv_heads) * case["dim"]
        most = 56 * 52 * 48 * 128
        if size > most:
            case.update(q_heads=8, kv_heads=8 if case["dim"] < 256 else 2)
        return case
    groups = rng.choice([1, 1, _spread(rng, 2, 8)])
    seqs = _spread(rng, 2, max(2, 64 // groups))
    chunk = rng.choice([1, 1, rng.randint(2, 12)])
    if seqs * groups * chunk > 128:
        chunk = 1
    case.update(groups=groups, seqs=seqs, chunk=chunk, alone=rng.random() < 0.3)
    # tokens x columns x dim within the largest listed case's
    most = 64 * 32 * 128 * 17000 / (groups * seqs * chunk * q_heads * case["dim"])
    shared = _spread(rng, 20, max(20, int(min(most * 0.9, 30000 / groups))))
    high = _spread(rng, 1, max(1, min(int(most * 0.1), 2000, 64 * 562 * 8 * 128 // (groups * seqs * kv_heads * case["dim"]))))
    case.update(shared=shared, low=int(high * rng.choice([0.01, 0.5, 1.0])), high=high)
    return case


# ---- the record of a block ------------------------------------------------------------------------------------------
# keys:   chunk of 32 dims | token % 8 | dim / 8 % 4 | token / 8 | dim % 8
# values: chunk of 32 dims | dim / 4 % 8 | token / 2 % 4 | dim % 4 | token / 8 | token % 2
def _codes_of(rec, D):
    """uint8 [..., 32 D + 16] -> codes float32 [..., 16, D] of keys and of values."""
    n, lead = rec.dim() - 1, rec.shape[:-1]
    k = rec[..., :16 * D].reshape(*lead, D // 32, 8, 4, 2, 8).permute(*range(n), n + 3, n + 1, n, n + 2, n + 4)
    v = rec[..., 16 * D:32 * D].reshape(*lead, D // 32, 8, 4, 4, 2, 2).permute(*range(n), n + 4, n + 2, n + 5, n, n + 1, n + 3)
    return k.reshape(*lead, BLOCK, D).float() - 128, v.reshape(*lead, BLOCK, D).float() - 128


def _scales_of(rec, D):
    """float32 [..., 2]: keys, values."""
    return rec[..., 32 * D:32 * D + 8].contiguous().view(torch.float32)


def _record(keys, values, scales, D):
    """codes [..., 16, D] and scales [..., 2] -> uint8 [..., 32 D + 16]."""
    lead, n = keys.shape[:-2], keys.dim() - 2
    k = (keys + 128).to(torch.uint8).reshape(*lead, 2, 8, D // 32, 4, 8).permute(*range(n), n + 2, n + 1, n + 3, n, n + 4)
    v = (values + 128).to(torch.uint8).reshape(*lead, 2, 4, 2, D // 32, 8, 4).permute(*range(n), n + 3, n + 4, n + 1, n + 5, n, n + 2)
    pair = torch.cat([scales, torch.zeros_like(scales)], -1).contiguous().view(torch.uint8)
    return torch.cat([k.reshape(*lead, 16 * D), v.reshape(*lead, 16 * D), pair], -1)


def _scale_for(amax):
    """The smallest power of two s, 2^-126 at least, with amax <= 127 s; 0 for 0."""
    m, e = torch.frexp(amax.double())  # amax = m 2^e, 0.5 <= m < 1
    e = torch.where(m <= 127 / 128, e - 7, e - 6).clamp(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(m), e), torch.zeros_like(m)).float()


# ---- what a program has in hand -------------------------------------------------------------------------------------
def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return out


def _cache(pages, H, P, D, channel, g):
    """Records of random keys (some channels larger than others) and values; blocks differ in size."""
    cache = torch.empty((pages, H, P // BLOCK, 32 * D + 16), dtype=torch.uint8, device=DEVICE)
    step = max(1, (1 << 27) // (H * P * D))
    for at in range(0, pages, step):
        n = min(step, pages - at)
        x = torch.randn((2, n, H, P // BLOCK, BLOCK, D), device=DEVICE, generator=g)
        x[0] *= channel[:, :, None]
        s = _scale_for(x.abs().amax((-1, -2)))
        x = torch.round(x / s[..., None, None])
        cache[at:at + n] = _record(x[0], x[1], torch.stack([s[0], s[1]], -1), D)
    return cache


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(DEVICE).manual_seed(seed)
    return {"append": _prepare_append, "attend": _prepare_attend, "score": _prepare_score}[case["op"]](case, host, g)


def _prepare_append(case, host, g):
    S, H, D, P = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    pick = lambda of, lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=of))  # noqa: E731
    fixed = torch.Generator().manual_seed(case["seqs"] + 100 * case["high"] + case["chunk"])
    # How many rows a sequence has, and where in its block it goes on, is the case's; how many blocks lie before that the seed's.
    rows, before = [], []
    for _ in range(S):
        rows.append(case["chunk"] if case["chunk"] == 1 or S == 1 else pick(fixed, 1, case["chunk"]))
        n = pick(fixed, case["low"], case["high"])
        before.append(n - BLOCK * pick(host, 0, (n - case["low"]) // BLOCK))
    if case["idle"]:
        rows[S // 2] = 0  # a slot without a token in this step
    width = max(1, max(-(-(b + n) // P) for b, n in zip(before, rows)))
    pages, total = S * width + 3, sum(rows) + (3 if case["idle"] else 0)
    channel = torch.exp(0.7 * torch.randn((H, 1, D), device=DEVICE, generator=g))
    cache = _cache(pages, H, P, D, channel, g)
    table = torch.randperm(pages, device=DEVICE, generator=g)[:S * width].to(torch.int32).reshape(S, width)
    # one buffer of all projections' rows, as a step keeps it: q, k and v are slices of its rows
    Q = case["q_heads"]
    qkv = torch.randn((total, Q + 2 * H, D), device=DEVICE, generator=g)
    qkv[:, Q:-H] *= channel[:, 0]
    qkv = qkv.to(getattr(torch, case["dtype"]))
    # A picture takes as many positions as its longer side, so positions lag behind slots.  Text has the same position on all
    # axes; a picture's rows share the time and go through height and width.
    places = torch.zeros((total, 3), dtype=torch.int64)
    for i, (a, n) in enumerate(zip(_starts(rows), rows)):
        p0, j = before[i] - before[i] // 3 - pick(host, 0, before[i] // 4), torch.arange(n)
        if case["grid"]:
            places[a:a + n] = p0 + torch.stack([torch.zeros_like(j), j // case["grid"], j % case["grid"]], -1)
        else:
            places[a:a + n] = p0 + j[:, None]
    # the axes take turns among the fast pairs, the slow ones are the time's
    axis = torch.arange(D // 2) % 3
    axis[3 * (D // 8):] = 0
    first = [b - b % BLOCK for b in before]  # every token of the blocks that the new rows fall in, for reading them back
    seen = [b + n - f if n else 0 for b, n, f in zip(before, rows, first)]
    k_read, v_read = torch.zeros((2, max(1, sum(seen)), H, D), dtype=torch.float16, device=DEVICE)
    return dict(op="append", cache=cache, table=table, row_start=_int32(_starts(rows)), lengths=_int32(before), D=D, H=H,
                q=qkv[:, :Q], k=qkv[:, Q:-H], v=qkv[:, -H:], positions=places.int().to(DEVICE), axis=axis.to(torch.uint8).to(DEVICE),
                inv_freq=1e6 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=DEVICE) / D),
                weights=[1 + 0.2 * torch.randn(D, device=DEVICE, generator=g) if case["norm"] else None for _ in range(2)],
                q_out=torch.zeros((total, Q, D), dtype=torch.float16, device=DEVICE),
                read_start=_int32(_starts(seen)), read_lengths=_int32(first), blocks=max(1, max(-(-n // BLOCK) for n in seen)), k_read=k_read, v_read=v_read)


def _prepare_attend(case, host, g):
    H, D, P, Q, N = case["kv_heads"], case["dim"], case["page"], case["q_heads"], case["groups"]
    pick = lambda of, lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=of))  # noqa: E731
    fixed = torch.Generator().manual_seed(N + 10 * case["seqs"] + 1000 * case["shared"] + case["chunk"])
    # The rows of each sequence are the case's; the lengths of prompts and answers the seed's.  What a group shares is whole pages.
    prompts = [max(1, (case["shared"] if N == 1 else pick(host, case["shared"] // 6, case["shared"])) // P) for _ in range(N)]
    groups = [0] * case["alone"]  # groups' sequences stand together; those in none before them
    groups += [i for i in range(N) for _ in range(case["seqs"])]
    rows, before = [], []
    for i, n in enumerate(groups):
        rows.append(1 if case["chunk"] == 1 else pick(fixed, 1, case["chunk"]))
        before.append(pick(host, case["low"], case["high"]) + prompts[n] * P)
    if case["idle"]:
        before[len(before) // 2] = -case["chunk"]  # a slot without a sequence: its rows see nothing
    # as wide as any seed's need be
    width = max(case["shared"] // P, 1) + -(-(case["high"] + case["chunk"]) // P)
    own_width = width - min(prompts)
    pages = sum(prompts) + len(groups) * own_width + case["alone"] * prompts[0] + 3
    channel = torch.exp(0.7 * torch.randn((H, 1, D), device=DEVICE, generator=g))
    cache = _cache(pages, H, P, D, channel, g)
    free = torch.randperm(pages, device=DEVICE, generator=g).to(torch.int32)
    table, at = torch.full((len(groups), width), -1, dtype=torch.int32, device=DEVICE), 0
    common = []
    for n in prompts:
        common.append(free[at:at + n])
        at += n
    for i, n in enumerate(groups):
        lone, have = i < case["alone"], -(-max(0, before[i] + rows[i]) // P)
        if not lone:
            table[i, :prompts[n]] = common[n]
        begin = 0 if lone else prompts[n]
        if have > begin:
            table[i, begin:have] = free[at:at + have - begin]
            at += have - begin
    total = sum(rows) + (3 if case["idle"] else 0)
    group_start = [case["alone"] + i * case["seqs"] for i in range(N + 1)]
    s = dict(op="attend", cache=cache, table=table, row_start=_int32(_starts(rows)), lengths=_int32(before), group_start=_int32(group_start),
             shared=_int32([n * P for n in prompts]), D=D, H=H, G=Q // H, most=max(rows), spans=[(i, i + 1, 0) for i in range(case["alone"])],
             q=torch.randn((total, Q, D), device=DEVICE, generator=g).half(), out=torch.zeros((total, Q, D), dtype=torch.float16, device=DEVICE))
    # (first sequence, the one behind the last, pages that they share)
    s["spans"] += [(a, b, n) for a, b, n in zip(group_start, group_start[1:], prompts)]
    if own:
        from paper_2609_35465_b200 import tetra
        s["workspace"] = tetra.tetra_kv_shared_workspace(D, total, Q, H, N)
    return s


def _prepare_score(case, host, g):
    R, V = case["rows"], case["vocab"]
    rnd = lambda *shape: torch.rand(shape, device=DEVICE, generator=g)  # noqa: E731
    # logits of a trained head: a broad bulk and a few tokens far above it; the given tokens are mostly among those
    x = 2.5 * torch.randn((R, V), device=DEVICE, generator=g)
    at = torch.randint(0, V, (R, 24), device=DEVICE, generator=g)
    x.scatter_add_(1, at, 6 + 7 * rnd(R, 24))
    tokens = at[:, :case["given"]].clone()
    far = rnd(R, case["given"]) < 0.2
    tokens = torch.where(far, torch.randint(0, V, tokens.shape, device=DEVICE, generator=g), tokens)
    f = lambda *shape: torch.zeros(shape, device=DEVICE)  # noqa: E731
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEVICE)  # noqa: E731
    return dict(op="score", logits=x.to(getattr(torch, case["dtype"])), tokens=tokens.int(), temperature=0.5 + rnd(R) if case["heated"] else None,
                logprob=f(R, case["given"]), rank=i(R, case["given"]), entropy=f(R), top_tokens=i(R, case["top"]) if case["top"] else None,
                top_logprob=f(R, case["top"]) if case["top"] else None)


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "attend": _attend, "score": _score}[s["op"]](s)


def _run_own(s):
    from paper_2609_35465_b200 import tetra
    if s["op"] == "append":
        tetra.tetra_kv_append_at(s["q"], s["k"], s["v"], s["cache"], s["table"], s["row_start"], s["lengths"], s["positions"], s["axis"], s["q_out"],
                                 s["inv_freq"], q_weight=s["weights"][0], k_weight=s["weights"][1], eps=1e-6)
        tetra.tetra_kv_read(s["cache"], s["table"], s["read_start"], s["read_lengths"], s["k_read"], s["v_read"])
        return dict(q=s["q_out"], k=s["k_read"], v=s["v_read"])
    if s["op"] == "attend":
        return tetra.tetra_kv_attend_shared(s["q"], s["cache"], s["table"], s["row_start"], s["lengths"], s["group_start"], s["shared"], s["out"], s["workspace"])
    tetra.tetra_logprobs(s["logits"], s["tokens"], s["logprob"], rank=s["rank"], entropy=s["entropy"], top_tokens=s["top_tokens"],
                         top_logprob=s["top_logprob"], temperature=s["temperature"])
    return _scores(s["logprob"], s["rank"], s["entropy"], s["top_tokens"], s["top_logprob"])


def _scores(logprob, rank, entropy, top_tokens, top_logprob):
    out = dict(logprob=logprob, rank=rank, entropy=entropy)
    return out if top_tokens is None else dict(out, top_tokens=top_tokens, top_logprob=top_logprob)


def _rows(starts, total):
    """For each of `total` rows: its sequence, its place among the sequence's rows, whether it belongs to any."""
    r = torch.arange(total, device=DEVICE)
    seq = torch.searchsorted(starts[1:].long(), r, right=True)
    live = seq < starts.numel() - 1
    seq = seq.clamp(max=starts.numel() - 2)
    return seq, r - starts[seq], live


def _turned(x, weight, angle):
    """Head norm (where there is a weight) and rotation by halves, in 64 bits: a key that lies next to the border of two codes is held to the right one."""
    x = x.double()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _append(s):
    D, H, cache, table = s["D"], s["H"], s["cache"], s["table"].long()
    S, B = table.shape[0], cache.shape[2]
    seq, i, live = _rows(s["row_start"], s["q"].shape[0])
    slot = s["lengths"][seq] + i
    angle = s["positions"][:, s["axis"].long()].double() * s["inv_freq"]
    q = (_turned(s["q"], s["weights"][0], angle) * live[:, None, None]).half()
    new = torch.stack([_turned(s["k"], s["weights"][1], angle).float(), s["v"].float()])  # [2, rows, H, D]
    # the blocks that each sequence's rows fall in: [S, blocks, H, record]
    first = s["lengths"].long() // BLOCK
    blocks = first[:, None] + torch.arange(s["blocks"], device=DEVICE)
    count = s["row_start"][1:] - s["row_start"][:-1]
    used = (blocks * BLOCK < (s["lengths"] + count)[:, None]) & (count > 0)[:, None]
    page = table.gather(1, (blocks // B).clamp(max=table.shape[1] - 1))
    place = blocks % B
    rec = cache[page, :, place]
    codes = torch.stack(_codes_of(rec, D))  # [2, S, blocks, H, 16, D]
    scale = _scales_of(rec, D).movedim(-1, 0)
    old = (blocks * BLOCK)[..., None] + torch.arange(BLOCK, device=DEVICE) < s["lengths"][:, None, None]  # [S, blocks, 16]
    scale = scale * old[..., 0, None]
    fill = torch.zeros_like(codes).transpose(3, 4).reshape(2, S, -1, H, D)  # the new rows at their places
    fill[:, seq[live], (slot - first[seq] * BLOCK)[live]] = new[:, live]
    fill = fill.reshape(2, S, s["blocks"], BLOCK, H, D).transpose(3, 4)
    grown = torch.maximum(scale, _scale_for(fill.abs().amax((-1, -2))))
    by = torch.where(grown > 0, grown, torch.ones_like(grown))[..., None, None]
    codes = torch.where(old[None, :, :, None, :, None], torch.round(codes * (scale[..., None, None] / by)), torch.round(fill / by))
    cache[page[used], :, place[used]] = _record(codes[0], codes[1], torch.stack([grown[0], grown[1]], -1), D)[used]
    # back to the rows of the reading
    values = (codes * grown[..., None, None]).half().transpose(3, 4).reshape(2, S, -1, H, D)
    rseq, ri, _ = _rows(s["read_start"], s["k_read"].shape[0])
    return dict(q=q, k=values[0, rseq, ri], v=values[1, rseq, ri])


def _tokens_of(s, pages):
    """Keys and values float32 [sequences, H, tokens, D] of page numbers [sequences, pages] (none: zeros)."""
    rec = s["cache"][pages.long().clamp(min=0)].transpose(2, 3)  # [S, pages, blocks, H, record]
    rec = rec.reshape(pages.shape[0], -1, s["H"], rec.shape[-1]).transpose(1, 2)
    scale = _scales_of(rec, s["D"])
    return [(c * scale[..., w, None, None]).reshape(pages.shape[0], s["H"], -1, s["D"]) for w, c in enumerate(_codes_of(rec, s["D"]))]


def _attend(s):
    """Group by group: the scores of all of its rows against the prompt, of each sequence's against its own tokens."""
    D, H, G, R, P = s["D"], s["H"], s["G"], s["most"], s["cache"].shape[2] * BLOCK
    seq, i, live = _rows(s["row_start"], s["q"].shape[0])
    S = s["table"].shape[0]
    q = torch.zeros((S, R, H, G, D), device=DEVICE)
    q[seq[live], i[live]] = s["q"][live].float().reshape(-1, H, G, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(S, H, R * G, D) / math.sqrt(D)
    last = (s["lengths"][:, None] + torch.arange(R, device=DEVICE)).repeat_interleave(G, 1)  # [S, R G]
    out = torch.zeros_like(q)
    for a, b, n in s["spans"]:
        k, v = _tokens_of(s, s["table"][a:b, n:])
        parts = [q[a:b] @ k.transpose(-1, -2)]
        if n:
            kp, vp = _tokens_of(s, s["table"][a:a + 1, :n])
            x = q[a:b].transpose(0, 1).reshape(1, H, -1, D) @ kp.transpose(-1, -2)
            parts.insert(0, x.reshape(H, b - a, R * G, -1).transpose(0, 1))
        x = torch.cat(parts, -1)
        x = x.masked_fill((torch.arange(x.shape[-1], device=DEVICE) > last[a:b, :, None])[:, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))
        out[a:b] = p[..., n * P:] @ v
        if n:
            x = p[..., :n * P].transpose(0, 1).reshape(1, H, -1, n * P) @ vp
            out[a:b] += x.reshape(H, b - a, R * G, D).transpose(0, 1)
    out = out.reshape(S, H, R, G, D).permute(0, 2, 1, 3, 4).reshape(S, R, H * G, D)
    return (out[seq, i.clamp(max=R - 1)] * live[:, None, None]).half()


def _score(s):
    x = s["logits"].float()
    R, V = x.shape
    T = torch.ones(R, 1, device=DEVICE) if s["temperature"] is None else s["temperature"][:, None]
    top = x.amax(-1, keepdim=True)
    z = (x - top) / T
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    norm = torch.log(total)
    entropy = norm - (e * z).sum(-1, keepdim=True, dtype=torch.float64) / total
    t = s["tokens"].long()
    mine = x.gather(1, t)
    index = torch.arange(V, device=DEVICE)
    rank = [((x > mine[:, j:j + 1]) | ((x == mine[:, j:j + 1]) & (index < t[:, j:j + 1]))).sum(-1) for j in range(t.shape[1])]
    logprob = lambda v: ((v - top) / T - norm).float()  # noqa: E731
    out = [logprob(mine), torch.stack(rank, -1).int(), entropy[:, 0].float(), None, None]
    if s["top_tokens"] is not None:
        n = s["top_tokens"].shape[1]
        most, at = torch.sort(x, dim=-1, descending=True, stable=True)
        out[3:] = at[:, :n].int(), logprob(most[:, :n])
    return _scores(*out)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------
def _places(D):
    """Byte of (token, dim) in a record's keys and in its values, as int64 [16, D]."""
    t, d = torch.arange(BLOCK, device=DEVICE)[:, None], torch.arange(D, device=DEVICE)[None]
    keys = d // 32 * 512 + (t % 8 * 4 + d % 32 // 8) * 16 + t // 8 * 8 + d % 8
    values = d // 32 * 512 + (d % 32 // 4 * 4 + t % 8 // 2) * 16 + d % 4 * 4 + t // 8 * 2 + t % 2
    return keys, 16 * D + values


def _context(s, i, n):
    """Keys and values of the first n tokens of sequence i, float64 [H, n, D]."""
    D, P = s["D"], s["cache"].shape[2] * BLOCK
    at = s["table"][i, :-(-n // P)].long()
    rec = s["cache"][at].transpose(0, 1).reshape(s["H"], -1, 32 * D + 16)
    scales = rec[..., 32 * D:32 * D + 8].contiguous().view(torch.float32).double()
    out = []
    for which, place in enumerate(_places(D)):
        codes = rec[:, :, place.reshape(-1)].double().sub_(128).reshape(*rec.shape[:2], BLOCK, D)
        out.append(codes.mul_(scales[..., which, None, None]).reshape(s["H"], -1, D)[:, :n])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "score": _exact_score}[case["op"]](s)


def _exact_attend(s):
    """Sequence by sequence, each with a context of its own."""
    D, H, G = s["D"], s["H"], s["G"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    starts, before = s["row_start"].tolist(), s["lengths"].tolist()
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        n = before[i] + b - a
        if n <= 0:
            continue
        k, v = _context(s, i, n)
        for r in range(a, b):
            m = before[i] + r - a + 1
            if m > 0:
                z = s["q"][r].double().reshape(H, G, D) @ k[:, :m].transpose(1, 2) / math.sqrt(D)
                out[r] = (torch.softmax(z, -1) @ v[:, :m]).reshape(H * G, D)
    return out


def _exact_append(s):
    """Sequence by sequence and block by block; a pair as a complex number."""
    D, H = s["D"], s["H"]
    starts, before = s["row_start"].tolist(), s["lengths"].tolist()
    q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    keys, values = [], []

    def turned(x, w, a, b):
        x = x[a:b].double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * w.double()
        phase = torch.stack([s["positions"][a:b, int(axis)] * f for axis, f in zip(s["axis"].tolist(), s["inv_freq"])], -1)
        z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * torch.polar(torch.ones_like(phase), phase)[:, None]
        return torch.cat([z.real, z.imag], -1)

    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        if a == b:
            continue
        q[a:b] = turned(s["q"], s["weights"][0], a, b)
        new = [turned(s["k"], s["weights"][1], a, b).float().double().transpose(0, 1), s["v"][a:b].double().transpose(0, 1)]
        lead = before[i] % BLOCK
        had = [x[:, before[i] - lead:] for x in _context(s, i, before[i])] if lead else [new[0][:, :0]] * 2
        block = before[i] // BLOCK
        page = s["table"][i, block // s["cache"].shape[2]].long()
        scales = s["cache"][page, :, block % s["cache"].shape[2], 32 * D:32 * D + 8].contiguous().view(torch.float32).double()
        for which, (o, n, out) in enumerate(zip(had, new, (keys, values))):
            every = torch.cat([o, n], 1)
            for at in range(0, every.shape[1], BLOCK):
                x = every[:, at:at + BLOCK]
                fresh = n[:, max(0, at - lead):at + BLOCK - lead].abs().amax((1, 2))
                scale = torch.where(fresh > 0, torch.exp2(torch.ceil(torch.log2(fresh / 127))), torch.zeros_like(fresh))
                if at == 0 and lead:
                    scale = torch.maximum(scale, scales[:, which])
                scale = scale[:, None, None]
                out.append((torch.round(x / torch.where(scale > 0, scale, torch.ones_like(scale))) * scale).transpose(0, 1))
    return dict(q=q, k=torch.cat(keys), v=torch.cat(values))


def _exact_score(s):
    """Some rows at a time; an order of whole numbers: the logit's, then the smaller index."""
    R, V = s["logits"].shape
    n = 0 if s["top_tokens"] is None else s["top_tokens"].shape[1]
    parts = []
    for a in range(0, R, 64):
        x = s["logits"][a:a + 64].double()
        if s["temperature"] is not None:
            x = x / s["temperature"][a:a + 64, None].double()
        lp = x - torch.logsumexp(x, -1, keepdim=True)
        bits = (s["logits"][a:a + 64].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * V + torch.arange(V - 1, -1, -1, device=DEVICE)
        t = s["tokens"][a:a + 64].long()
        mine = order.gather(1, t)
        first = order.topk(max(n, 1), -1)[1]
        parts.append((lp.gather(1, t), torch.stack([(order > mine[:, j:j + 1]).sum(-1) for j in range(t.shape[1])], -1),
                      -(lp.exp() * lp).sum(-1), first[:, :n], lp.gather(1, first[:, :n])))
    lp, rank, entropy, top, top_lp = (torch.cat(p) for p in zip(*parts))
    return _scores(lp, rank.int(), entropy, top.int() if n else None, top_lp)


def work(case):
    if case["op"] == "score":
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * (4 if case["dtype"] == "float32" else 2) + case["rows"] * (12 * case["given"] + 8 * case["top"] + 4), flops=6 * n)
    heads, H, D, S = case["q_heads"], case["kv_heads"], case["dim"], case["seqs"]
    rows = S * (case["chunk"] if case["chunk"] == 1 or S == 1 else (1 + case["chunk"]) / 2)
    per = (32 * D + 16) / BLOCK * H  # a token of the cache
    if case["op"] == "append":
        size = 4 if case["dtype"] == "float32" else 2
        # rows in, queries out, their blocks written, and those read and written as float16
        return dict(bytes=rows * D * ((heads + 2 * H) * size + heads * 2) + (rows + 8 * S) * (2 * per + 4 * D * H), flops=rows * D * (heads + H) * 10)
    N = case["groups"]
    prompt = case["shared"] * (1 if N == 1 else 7 / 12)
    tail = (case["low"] + case["high"]) / 2
    rows = N * S * (1 if case["chunk"] == 1 else (1 + case["chunk"]) / 2) + case["alone"]
    tokens = N * (prompt + S * tail) + case["alone"] * (prompt + tail)
    return dict(bytes=tokens * per + rows * heads * D * 4, flops=4 * (prompt + tail) * rows * heads * D)
