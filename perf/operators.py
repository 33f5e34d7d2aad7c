"""The operators that stand between a decode step's products, as cases that can be timed and compared: a paged cache of
keys and values in 8 bits that grows, the attention over it, and the choice of the next token.

  append   projections of new tokens (head norm, rotation) into the cache, and the blocks they fell in read back:
           tetra_kv_append + tetra_kv_read
  attend   attention of single tokens or short chunks over the cache: tetra_kv_attend
  sample   next tokens from the output head's logits: tetra_sample

The cache holds, for each page, kv head and block of 16 tokens, a record of 32 D + 16 bytes: 16 D bytes of keys, 16 D of
values (code + 128; the orders stand above `_keys_of`), one float32 scale for the keys, one for the
values, and eight bytes without meaning; a scale is a power of two.  `row_start` says which rows belong to which sequence,
`lengths` how many tokens each sequence had before these rows.

Shapes are those of shapes.py (dense models with 32 or 40 query heads and 8 kv heads of 128, a vocabulary of 151936) and
generic sizes around them.
"""
import math

import torch

own = False

DEVICE = "cuda"
BLOCK = 16
WORKSPACE = 32 << 20  # bytes that a program keeps for tetra_kv_attend, zeroed once


def listed():
    return [
        # one token of one 8B sequence appended: the step of a chat, latency is all there is
        dict(name="append_1_8b", op="append", seqs=1, chunk=1, low=700, high=700, q_heads=32, kv_heads=8, dim=128, page=64, dtype="float32", norm=True, idle=False),
        # a server's batch of the 14B model, ragged lengths, one slot without a token, padded to a fixed batch
        dict(name="append_64_14b", op="append", seqs=64, chunk=1, low=1, high=900, q_heads=40, kv_heads=8, dim=128, page=32, dtype="float32", norm=True, idle=True),
        # pieces of prompts, 16 rows at most to a piece (as many as a product takes), half precision, small heads
        dict(name="append_chunks_64", op="append", seqs=12, chunk=16, low=0, high=333, q_heads=16, kv_heads=2, dim=64, page=16, dtype="float16", norm=False, idle=False),
        # the first tokens of a chat, one sequence
        dict(name="attend_1x257_8b", op="attend", seqs=1, chunk=1, low=257, high=257, q_heads=32, kv_heads=8, dim=128, page=64, idle=False),
        # one sequence with a long document before it
        dict(name="attend_1x40961_8b", op="attend", seqs=1, chunk=1, low=40961, high=40961, q_heads=32, kv_heads=8, dim=128, page=64, idle=False),
        # a server's batch of the 14B model (five query heads to a kv head), ragged, one slot without a sequence
        dict(name="attend_16_ragged_14b", op="attend", seqs=16, chunk=1, low=1, high=4000, q_heads=40, kv_heads=8, dim=128, page=32, idle=True),
        # the largest batch: 64 sequences of up to 8192 tokens
        dict(name="attend_64x8192_8b", op="attend", seqs=64, chunk=1, low=7000, high=8192, q_heads=32, kv_heads=8, dim=128, page=128, idle=False),
        # pieces of prompts behind a context, up to 16 rows to a piece, causal among themselves
        dict(name="attend_chunks_8b", op="attend", seqs=4, chunk=16, low=500, high=6001, q_heads=32, kv_heads=8, dim=128, page=16, idle=False),
        # one token of one sequence, the usual settings
        dict(name="sample_1_head", op="sample", rows=1, vocab=151936, dtype="float32", temperature=0.7, top_k=20, top_p=0.8, min_p=0.0, mixed=False),
        # a small vocabulary of odd size in half precision (many equal logits), each row with settings of its own
        dict(name="sample_7x32003", op="sample", rows=7, vocab=32003, dtype="float16", temperature=1.0, top_k=50, top_p=0.9, min_p=0.02, mixed=True),
        # a server's batch, only the mass counts: no fixed number of candidates
        dict(name="sample_16_nucleus", op="sample", rows=16, vocab=151936, dtype="float32", temperature=1.0, top_k=0, top_p=0.95, min_p=0.0, mixed=False),
        # the largest batch, each row with settings of its own
        dict(name="sample_64_mixed", op="sample", rows=64, vocab=151936, dtype="float32", temperature=0.8, top_k=40, top_p=0.9, min_p=0.05, mixed=True),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "sample", "attend"])
    if op == "sample":
        vocab = _spread(rng, 500, 262144)
        return dict(op=op, rows=min(_spread(rng, 1, 64), max(1, 64 * 151936 // vocab)), vocab=vocab, dtype=rng.choice(["float32", "float16"]),
                    temperature=round(rng.uniform(0.3, 1.6), 3), top_k=rng.choice([0, 0, 1, 20, _spread(rng, 2, 2000)]),
                    top_p=rng.choice([1.0, round(rng.uniform(0.1, 0.99), 3)]), min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.3), 3)]),
                    mixed=rng.random() < 0.5)
    q_heads, kv_heads = rng.choice([(32, 8), (40, 8), (16, 2), (8, 8), (7, 1), (24, 2)])
    case = dict(op=op, q_heads=q_heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128, 128, 256]), page=rng.choice([16, 32, 48, 64, 128]),
                seqs=_spread(rng, 1, 64), chunk=rng.choice([1, 1, 1, rng.randint(2, 16)]), idle=rng.random() < 0.3)
    case["idle"] = case["idle"] and case["seqs"] > 1
    if op == "append":
        high = _spread(rng, 1, 1000)
        case.update(low=rng.randint(0, high), high=high, dtype=rng.choice(["float32", "float16"]), norm=rng.random() < 0.5)
        case["seqs"] = min(case["seqs"], max(1, 256 // case["chunk"]))
        return case
    # tokens x kv heads x dim, and rows with them, within the largest listed case's
    rows = 1 if case["chunk"] == 1 else case["chunk"] * (q_heads // kv_heads) / 4
    most = int(64 * 8192 * 8 * 128 / (case["seqs"] * kv_heads * case["dim"] * rows))
    high = _spread(rng, 1, max(1, min(most, 100000)))
    case.update(low=max(1, int(high * rng.choice([0.01, 0.5, 1.0]))), high=high)
    return case


# ---- the record of a block ------------------------------------------------------------------------------------------
# keys:   chunk of 32 dims | token % 8 | dim / 8 % 4 | token / 8 | dim % 8
# values: chunk of 32 dims | dim / 4 % 8 | token / 2 % 4 | dim % 4 | token / 8 | token % 2
def _keys_of(part, D):
    """uint8 [..., 16 D] -> codes float32 [..., 16, D]."""
    n = part.dim() - 1
    x = part.reshape(*part.shape[:-1], D // 32, 8, 4, 2, 8).permute(*range(n), n + 3, n + 1, n, n + 2, n + 4)
    return x.reshape(*part.shape[:-1], BLOCK, D).float() - 128


def _values_of(part, D):
    n = part.dim() - 1
    x = part.reshape(*part.shape[:-1], D // 32, 8, 4, 4, 2, 2).permute(*range(n), n + 4, n + 2, n + 5, n, n + 1, n + 3)
    return x.reshape(*part.shape[:-1], BLOCK, D).float() - 128


def _scales_of(records, D):
    """float32 [..., 2]: keys, values."""
    return records[..., 32 * D:32 * D + 8].contiguous().view(torch.float32)


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
def _counts(case, g):
    """(rows, tokens before them) of each sequence, on the host.  How many rows there are, and where in its block a sequence
    goes on, is the case's; how many blocks lie before that, or how many tokens the attention has before it, is the seed's."""
    rows, before = [], []
    fixed = torch.Generator().manual_seed(case["seqs"] + 100 * case["high"] + case["chunk"])
    pick = lambda of, lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=of))  # noqa: E731
    for i in range(case["seqs"]):
        rows.append(1 if case["chunk"] == 1 else pick(fixed, 1, case["chunk"]))
        n = pick(fixed, case["low"], case["high"])
        if case["op"] == "append":
            before.append(n - BLOCK * pick(g, 0, (n - case["low"]) // BLOCK))
        else:
            before.append(max(0, pick(g, case["low"], case["high"]) - rows[-1]))
    if case["idle"]:
        if case["op"] == "append":
            rows[len(rows) // 2] = 0      # a slot without a token in this step
        else:
            before[len(before) // 2] = -case["chunk"]  # a slot without a sequence: its rows see nothing
    return rows, before


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return _int32(out)


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(DEVICE).manual_seed(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, g)
    S, H, D, P = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    rows, before = _counts(case, host)
    width = max(1, max(-(-max(0, b + n) // P) for b, n in zip(before, rows)))
    pages = S * width + 3
    # keys have channels that are larger than others, values are even; blocks differ in size
    channel = torch.exp(0.7 * torch.randn((H, 1, D), device=DEVICE, generator=g))
    cache = torch.empty((pages, H, P // BLOCK, 32 * D + 16), dtype=torch.uint8, device=DEVICE)
    step = max(1, (1 << 27) // (H * P * D))
    for at in range(0, pages, step):
        n = min(step, pages - at)
        x = torch.randn((2, n, P // BLOCK, H, BLOCK, D), device=DEVICE, generator=g)
        x[0] *= channel
        x = x.transpose(2, 3)
        s = _scale_for(x.abs().amax((-1, -2)))
        x = torch.round(x / s[..., None, None])
        cache[at:at + n] = _record(x[0], x[1], torch.stack([s[0], s[1]], -1), D)
    table = torch.randperm(pages, device=DEVICE, generator=g)[:S * width].to(torch.int32).reshape(S, width)
    spare = 3 if case["idle"] else 0
    total = sum(rows) + spare
    s = dict(op=case["op"], cache=cache, table=table, row_start=_starts(rows), lengths=_int32(before), D=D, H=H, G=case["q_heads"] // H, most=max(rows),
             q_out=torch.zeros((total, case["q_heads"], D), dtype=torch.float16, device=DEVICE))
    if case["op"] == "attend":
        s["q"] = torch.randn((total, case["q_heads"], D), device=DEVICE, generator=g).half()
        s["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device=DEVICE)
        return s
    kind = getattr(torch, case["dtype"])
    # one buffer of all projections' rows, as a step keeps it: q, k and v are slices of its rows
    qkv = torch.randn((total, case["q_heads"] + 2 * H, D), device=DEVICE, generator=g)
    qkv[:, case["q_heads"]:-H] *= channel[:, 0]
    qkv = qkv.to(kind)
    s.update(q=qkv[:, :case["q_heads"]], k=qkv[:, case["q_heads"]:-H], v=qkv[:, -H:])
    s["inv_freq"] = 1e6 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=DEVICE) / D)
    s["weights"] = [1 + 0.2 * torch.randn(D, device=DEVICE, generator=g) if case["norm"] else None for _ in range(2)]
    # every token of the blocks that the new rows fall in, for reading them back
    first = [b - b % BLOCK for b in before]
    seen = [b + n - f if n else 0 for b, n, f in zip(before, rows, first)]
    s.update(read_start=_starts(seen), read_lengths=_int32(first), blocks=max(-(-n // BLOCK) for n in seen) or 1)
    s["k_read"], s["v_read"] = torch.zeros((2, max(1, sum(seen)), H, D), dtype=torch.float16, device=DEVICE)
    return s


def _prepare_sample(case, g):
    R, V = case["rows"], case["vocab"]
    rnd = lambda *shape: torch.rand(shape, device=DEVICE, generator=g)  # noqa: E731
    # logits of a trained head: a broad bulk and a few tokens far above it
    x = 2.5 * torch.randn((R, V), device=DEVICE, generator=g)
    at = torch.randint(0, V, (R, 24), device=DEVICE, generator=g)
    x.scatter_add_(1, at, 6 + 7 * rnd(R, 24))
    full = lambda v, t: torch.full((R,), v, dtype=t, device=DEVICE)  # noqa: E731
    T, k, p, m = full(case["temperature"], torch.float32), full(case["top_k"], torch.int32), full(case["top_p"], torch.float32), full(case["min_p"], torch.float32)
    if case["mixed"]:
        off = rnd(4, R) < 0.3
        T = torch.where(off[0], torch.zeros_like(T), T * (0.5 + rnd(R)))   # 0: the largest logit
        k = torch.where(off[1], torch.zeros_like(k), (k * (0.5 + rnd(R))).int())
        p = torch.where(off[2], torch.ones_like(p), p * (0.8 + 0.2 * rnd(R)))
        m = torch.where(off[3], torch.zeros_like(m), m)
    return dict(op="sample", logits=x.to(getattr(torch, case["dtype"])), u=rnd(R), temperature=T, top_k=k, top_p=p, min_p=m,
                tokens=torch.zeros(R, dtype=torch.int32, device=DEVICE), prob=torch.zeros(R, device=DEVICE))


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "attend": _attend, "sample": _sample}[s["op"]](s)


def _run_own(s):
    from paper_2609_35465_b200 import tetra
    if s["op"] == "append":
        tetra.tetra_kv_append(s["q"], s["k"], s["v"], s["cache"], s["table"], s["row_start"], s["lengths"], s["q_out"],
                              inv_freq=s["inv_freq"], q_weight=s["weights"][0], k_weight=s["weights"][1], eps=1e-6)
        tetra.tetra_kv_read(s["cache"], s["table"], s["read_start"], s["read_lengths"], s["k_read"], s["v_read"])
        return dict(q=s["q_out"], k=s["k_read"], v=s["v_read"])
    if s["op"] == "attend":
        tetra.tetra_kv_attend(s["q"], s["cache"], s["table"], s["row_start"], s["lengths"], s["q_out"], s["workspace"])
        return s["q_out"]
    tetra.tetra_sample(s["logits"], s["u"], s["tokens"], prob=s["prob"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return dict(tokens=s["tokens"], prob=s["prob"])


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
    pos = s["lengths"][seq] + i
    angle = pos.double()[:, None] * s["inv_freq"]
    q = (_turned(s["q"], s["weights"][0], angle) * live[:, None, None]).half()
    new = torch.stack([_turned(s["k"], s["weights"][1], angle).float(), s["v"].float()])  # [2, rows, H, D]
    # the blocks that each sequence's rows fall in: [S, blocks, H, record]
    first = s["lengths"].long() // BLOCK
    blocks = first[:, None] + torch.arange(s["blocks"], device=DEVICE)
    fresh = s["row_start"][1:] > s["row_start"][:-1]
    used = (blocks * BLOCK < (s["lengths"] + s["row_start"][1:] - s["row_start"][:-1])[:, None]) & fresh[:, None]
    page = table.gather(1, (blocks // B).clamp(max=table.shape[1] - 1))
    place = blocks % B
    rec = cache[page, :, place]
    codes = torch.stack([_keys_of(rec[..., :16 * D], D), _values_of(rec[..., 16 * D:32 * D], D)])  # [2, S, blocks, H, 16, D]
    scale = _scales_of(rec, D).movedim(-1, 0)
    old = (blocks * BLOCK)[..., None] + torch.arange(BLOCK, device=DEVICE) < s["lengths"][:, None, None]  # [S, blocks, 16]
    scale = scale * old[..., 0, None]
    fill = torch.zeros_like(codes).transpose(3, 4).reshape(2, S, -1, H, D)  # the new rows at their places
    fill[:, seq[live], (pos - first[seq] * BLOCK)[live]] = new[:, live]
    fill = fill.reshape(2, S, s["blocks"], BLOCK, H, D).transpose(3, 4)
    grown = torch.maximum(scale, _scale_for(fill.abs().amax((-1, -2))))
    by = torch.where(grown > 0, grown, torch.ones_like(grown))[..., None, None]
    codes = torch.where(old[None, :, :, None, :, None], torch.round(codes * (scale[..., None, None] / by)), torch.round(fill / by))
    cache[page[used], :, place[used]] = _record(codes[0], codes[1], torch.stack([grown[0], grown[1]], -1), D)[used]
    # back to the rows of the reading
    values = (codes * grown[..., None, None]).half().transpose(3, 4).reshape(2, S, -1, H, D)
    rseq, ri, _ = _rows(s["read_start"], s["k_read"].shape[0])
    return dict(q=q, k=values[0, rseq, ri], v=values[1, rseq, ri])


def _attend(s):
    D, H, G, table = s["D"], s["H"], s["G"], s["table"].long()
    S, R = table.shape[0], s["most"]
    rec = s["cache"][table].transpose(2, 3)  # [S, pages, blocks, H, record]
    rec = rec.reshape(S, -1, H, rec.shape[-1]).transpose(1, 2)
    scale = _scales_of(rec, D)
    k = (_keys_of(rec[..., :16 * D], D) * scale[..., :1, None]).reshape(S, H, -1, D)
    seq, i, live = _rows(s["row_start"], s["q"].shape[0])
    q = torch.zeros((S, R, H, G, D), device=DEVICE)
    q[seq[live], i[live]] = s["q"][live].float().reshape(-1, H, G, D)
    x = (q.permute(0, 2, 1, 3, 4).reshape(S, H, R * G, D) / math.sqrt(D)) @ k.transpose(-1, -2)
    last = (s["lengths"][:, None] + torch.arange(R, device=DEVICE)).repeat_interleave(G, 1)  # [S, R G]
    seen = torch.arange(x.shape[-1], device=DEVICE) <= last[..., None]
    x = x.masked_fill(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    v = (_values_of(rec[..., 16 * D:32 * D], D) * scale[..., 1:, None]).reshape(S, H, -1, D)
    o = (p @ v).reshape(S, H, R, G, D).permute(0, 2, 1, 3, 4).reshape(S, R, H * G, D)
    return (o[seq, i.clamp(max=R - 1)] * live[:, None, None]).half()


def _weights(x, T):
    """exp((x - max) / T) in 64 bits, the largest's being 1; T 0: the first of the largest alone."""
    x = x.double()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top, first = x.max(-1, keepdim=True)
    first = (x == top).int().argmax(-1, keepdim=True)
    T = T.double()[:, None]
    e = torch.exp((x - top) / torch.where(T > 0, T, torch.ones_like(T)))
    alone = torch.zeros_like(e).scatter_(1, first, 1.0)
    return x, torch.where(T > 0, e, alone)


def _sample(s):
    x, e = _weights(s["logits"], s["temperature"])
    V = x.shape[1]
    order = torch.sort(x, dim=-1, descending=True, stable=True)[1]
    es, at = e.gather(1, order), torch.arange(V, device=DEVICE)
    k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    in_k = at < k
    es = torch.where(in_k, es, torch.zeros_like(es))
    cum = es.cumsum(-1)
    p = s["top_p"].double()[:, None]
    in_p = (cum - es < p * cum[:, -1:]) | (p >= 1)
    in_m = es >= s["min_p"].double()[:, None]
    keep = in_k & ((in_p & in_m) | (at == 0))
    w = torch.zeros_like(e).scatter_(1, order, torch.where(keep, es, torch.zeros_like(es)))
    cum = w.cumsum(-1)
    total = cum[:, -1:]
    token = (cum > s["u"].double()[:, None] * total).int().argmax(-1)
    return dict(tokens=token.int(), prob=(w.gather(1, token[:, None]) / total)[:, 0].float())


# ---- the definition in 64 bits, sequence by sequence ----------------------------------------------------------------
def _places(D):
    """Byte of (token, dim) in a record's keys and in its values, as int64 [16, D]."""
    t, d = torch.arange(BLOCK, device=DEVICE)[:, None], torch.arange(D, device=DEVICE)[None]
    keys = d // 32 * 512 + (t % 8 * 4 + d % 32 // 8) * 16 + t // 8 * 8 + d % 8
    values = d // 32 * 512 + (d % 32 // 4 * 4 + t % 8 // 2) * 16 + d % 4 * 4 + t // 8 * 2 + t % 2
    return keys, 16 * D + values


def _tokens(s, i, n):
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
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](s)


def _exact_attend(s):
    D, H, G = s["D"], s["H"], s["G"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    starts, before = s["row_start"].tolist(), s["lengths"].tolist()
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        n = before[i] + b - a
        if n <= 0:
            continue
        k, v = _tokens(s, i, n)
        for r in range(a, b):
            m = before[i] + r - a + 1
            if m > 0:
                z = s["q"][r].double().reshape(H, G, D) @ k[:, :m].transpose(1, 2) / math.sqrt(D)
                out[r] = (torch.softmax(z, -1) @ v[:, :m]).reshape(H * G, D)
    return out


def _exact_append(s):
    D, H = s["D"], s["H"]
    starts, before = s["row_start"].tolist(), s["lengths"].tolist()
    q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    keys, values = [], []

    def turned(x, w, pos):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * w.double()
        z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * torch.polar(torch.ones_like(s["inv_freq"]), pos * s["inv_freq"])
        return torch.cat([z.real, z.imag], -1)

    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        if a == b:
            continue
        for r in range(a, b):
            q[r] = turned(s["q"][r], s["weights"][0], before[i] + r - a)
        new = [torch.stack([turned(s["k"][r], s["weights"][1], before[i] + r - a).float().double() for r in range(a, b)]).transpose(0, 1), s["v"][a:b].double().transpose(0, 1)]
        first = before[i] - before[i] % BLOCK
        had = _tokens(s, i, before[i]) if before[i] else [torch.zeros((H, 0, D), dtype=torch.float64, device=DEVICE)] * 2
        page = s["table"][i, first // (s["cache"].shape[2] * BLOCK)].long()
        rec = s["cache"][page, :, first // BLOCK % s["cache"].shape[2]]
        scales = rec[:, 32 * D:32 * D + 8].contiguous().view(torch.float32).double()
        for which, (o, n, out) in enumerate(zip(had, new, (keys, values))):
            every = torch.cat([o[:, first:], n], 1)
            for at in range(0, every.shape[1], BLOCK):
                x = every[:, at:at + BLOCK]
                fresh = n[:, max(0, at - (before[i] - first)):at + BLOCK - (before[i] - first)].abs().amax((1, 2))
                scale = torch.where(fresh > 0, torch.exp2(torch.ceil(torch.log2(fresh / 127))), torch.zeros_like(fresh))
                if at == 0 and before[i] > first:
                    scale = torch.maximum(scale, scales[:, which])
                scale = scale[:, None, None]
                out.append((torch.round(x / torch.where(scale > 0, scale, torch.ones_like(scale))) * scale).transpose(0, 1))
    return dict(q=q, k=torch.cat(keys), v=torch.cat(values))


def _exact_sample(s):
    import numpy as np
    tokens, prob = [], []
    for r in range(s["logits"].shape[0]):
        x, T = s["logits"][r].double().cpu().numpy(), float(s["temperature"][r])
        k, p, m = int(s["top_k"][r]), float(s["top_p"][r]), float(s["min_p"][r])
        order = np.argsort(-x, kind="stable")
        w = np.exp((x[order] - x[order[0]]) / T) if T > 0 else (np.arange(x.size) == 0) * 1.0
        n = min(k, x.size) if k > 0 else x.size
        if p < 1:
            n = min(n, 1 + int(np.searchsorted(np.cumsum(w[:n]), p * w[:n].sum())))
        n = max(1, min(n, int((w >= m).sum())))
        kept = np.sort(order[:n])
        mass = np.zeros(x.size)
        mass[order[:n]] = w[:n]
        c = np.cumsum(mass[kept])
        at = kept[min(n - 1, int(np.searchsorted(c, float(s["u"][r]) * c[-1], side="right")))]
        tokens.append(int(at))
        prob.append(mass[at] / c[-1])
    return dict(tokens=torch.tensor(tokens, dtype=torch.int32), prob=torch.tensor(prob, dtype=torch.float64))


def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * (4 if case["dtype"] == "float32" else 2) + 24 * case["rows"], flops=4 * n)
    heads, D, S = case["q_heads"], case["dim"], case["seqs"]
    rows = S * (1 if case["chunk"] == 1 else (1 + case["chunk"]) / 2)
    if case["op"] == "append":
        size = 4 if case["dtype"] == "float32" else 2
        # rows in, queries out, a block of each head and sequence read and written, its tokens read and written as float16
        blocks = S * case["kv_heads"] * (32 * D + 16) * (1 + case["chunk"] / BLOCK / 2)
        return dict(bytes=rows * D * ((heads + 2 * case["kv_heads"]) * size + heads * 2) + 5 * blocks, flops=rows * D * (heads + case["kv_heads"]) * 10)
    tokens = S * (case["low"] + case["high"]) / 2
    per = (32 * D + 16) / BLOCK * case["kv_heads"]
    return dict(bytes=tokens * per + rows * heads * D * 4, flops=4 * tokens * (rows / S) * heads * D)
