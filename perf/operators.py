"""Timed cases of the paged KV cache: the append with the rotation on the way, the attention of a batch's new tokens over
the pages, and the way back out of the pages, each as a serving program calls it for one layer of one step.

The cache is a pool of pages.  A page holds `page` positions of every kv head, keys and values apart, in blocks of 32
positions: element (position p of the block, dim j) of a key block of bf16 lies at (j/8, p, j%8), of one in e4m3 at
(j/16, p, j%16); of a value block of bf16 at (2t + h, j, 4a + b) and in e4m3 at (h, j, 8t + 4a + b), where
p = 16t + 8a + 4h + b.  A table names the page of every `page` positions of a sequence; -1 stands for a page that is not
there, whose positions no query sees.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DEVICE = "cuda"

# query heads, kv heads, head dim, rotary base
SHAPES = {
    "tiny": (4, 4, 64, 10000.0),
    "7b": (32, 32, 128, 10000.0),
    "8b_gqa": (32, 8, 128, 500000.0),
    "13b": (40, 40, 128, 10000.0),
    "70b": (64, 8, 128, 500000.0),
}

# A case's keys: `prompts` sequences bring new_lo .. new_hi new tokens each on top of cached_lo .. cached_hi cached
# positions, `decodes` sequences bring one token on cache_lo .. cache_hi; the lengths come from the case alone (`lengths`).
# `window`: how many positions a query sees at most (0: all before it); pages that have left every query's window are gone.
NONE = {"e4m3": False, "page": 64, "window": 0, "prompts": 0, "new_lo": 0, "new_hi": 0, "cached_lo": 0, "cached_hi": 0,
        "decodes": 0, "cache_lo": 0, "cache_hi": 0, "lengths": 1}
K_SCALE, V_SCALE = 0.0137, 0.0121       # what one step of an e4m3 cache stands for: about the largest value over 448


def listed():
    def named(name, op, shape, **more):
        return dict(NONE, op=op, shape=shape, name=name, **more)

    return [
        # one user's answer: the new token's key and value, launch and latency only
        named("append_1", "append", "8b_gqa", decodes=1, cache_lo=1171, cache_hi=1171),
        # a full house of answers on an 8-bit cache
        named("append_161_e4m3", "append", "7b", e4m3=True, decodes=161, cache_lo=128, cache_hi=1024),
        # the benchmark's mixed batch: prompts and running answers, no grouped heads
        named("append_mixed_16_48", "append", "13b", prompts=16, new_lo=32, new_hi=2000, decodes=48, cache_lo=128, cache_hi=2048),
        # one user's answer
        named("decode_1", "attention", "8b_gqa", decodes=1, cache_lo=1171, cache_hi=1171),
        # the benchmark's continuous decode
        named("decode_64", "attention", "8b_gqa", decodes=64, cache_lo=256, cache_hi=4096),
        # long caches in 8 bits on the largest shape
        named("decode_32_e4m3", "attention", "70b", e4m3=True, page=128, decodes=32, cache_lo=512, cache_hi=12000),
        # drafted tokens being checked: a few new tokens per sequence
        named("draft_24", "attention", "8b_gqa", page=32, prompts=24, new_lo=3, new_hi=8, cached_lo=200, cached_hi=4000),
        # a chunk of a long prompt beside running answers
        named("chunk_512_decode_40", "attention", "8b_gqa", prompts=1, new_lo=512, new_hi=512, cached_lo=3001, cached_hi=3001,
              decodes=40, cache_lo=256, cache_hi=4096),
        # a sliding window over an 8-bit cache, old pages freed
        named("window_prompts_e4m3", "attention", "7b", e4m3=True, window=1000, prompts=3, new_lo=301, new_hi=777, cached_lo=1500,
              cached_hi=3001),
        # the benchmark's prefill batch on the largest shape
        named("prefill_4x2048", "attention", "70b", prompts=4, new_lo=2048, new_hi=2048),
        # a short answer handed over to another instance
        named("read_301", "read", "tiny", page=32, decodes=1, cache_lo=300, cache_hi=300),
        # a long conversation handed over out of an 8-bit cache
        named("read_16000_e4m3", "read", "13b", e4m3=True, page=128, decodes=1, cache_lo=16000, cache_hi=16000),
    ]


def _spread(rng, lo, hi):
    """A whole number, spread over the logarithm of the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    shape = rng.choice(["tiny", "7b", "8b_gqa", "8b_gqa", "13b", "70b"])
    case = dict(NONE, op=rng.choice(["append", "attention", "attention", "attention", "read"]), shape=shape, e4m3=rng.random() < 0.4,
                page=rng.choice([32, 64, 128, 256]), lengths=rng.randrange(1 << 20))
    heads, kv_heads, d, _ = SHAPES[shape]
    kind = rng.choice(["decode", "draft", "chunk", "prefill", "mixed"])
    if case["op"] == "read":
        n = _spread(rng, 20, 16000)
        return dict(case, decodes=1, cache_lo=n, cache_hi=n)
    if kind in ("decode", "mixed"):
        top = _spread(rng, 100, 8000)
        case.update(decodes=_spread(rng, 1, max(1, min(200, 1500000 // (kv_heads * top)))), cache_lo=top // 8, cache_hi=top)
    if kind == "draft":
        top = _spread(rng, 100, 6000)
        case.update(prompts=_spread(rng, 1, max(1, min(64, 1500000 // (kv_heads * top)))), new_lo=2, new_hi=rng.randint(3, 16),
                    cached_lo=top // 8, cached_hi=top)
    if kind in ("chunk", "mixed"):
        before, new = _spread(rng, 50, 6000), _spread(rng, 17, 1024)
        case.update(prompts=rng.randint(1, 3), new_lo=max(2, new // 3), new_hi=new, cached_lo=before // 2, cached_hi=before)
    if kind == "prefill":
        new = _spread(rng, 33, 2048)
        case.update(prompts=_spread(rng, 1, 8 if new < 1024 else 4), new_lo=max(2, new // 4), new_hi=new)
    if case["op"] == "attention" and rng.random() < 0.3:
        case["window"] = _spread(rng, 64, 4096)
    return case


def _lengths(case):
    """(new tokens, cached positions) of every sequence, prompts first."""
    rng = random.Random(case["lengths"])
    seqs = []
    for _ in range(case["prompts"]):
        seqs.append((_spread(rng, case["new_lo"], case["new_hi"]), rng.randint(case["cached_lo"], case["cached_hi"])))
    for _ in range(case["decodes"]):
        seqs.append((1, rng.randint(case["cache_lo"], case["cache_hi"])))
    return seqs


def prepare(case, seed):
    heads, kv_heads, d, base = SHAPES[case["shape"]]
    seqs, page = _lengths(case), case["page"]
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = SimpleNamespace(case=case, heads=heads, kv_heads=kv_heads, d=d, base=base, page=page, seqs=seqs, window=case["window"])
    s.new = [n for n, _ in seqs]
    s.before = [b for _, b in seqs]
    s.q_start = [sum(s.new[:i]) for i in range(len(seqs) + 1)]
    tokens = s.q_start[-1]
    # the projection of the batch: query, key and value heads of a token in one row
    row = (heads + 2 * kv_heads) * d
    s.qkv = torch.randn(tokens, row, generator=g, device=DEVICE).bfloat16()
    s.q, s.k, s.v = s.qkv[:, :heads * d], s.qkv[:, heads * d:(heads + kv_heads) * d], s.qkv[:, (heads + kv_heads) * d:]
    s.out = torch.empty(tokens, heads * d, dtype=torch.bfloat16, device=DEVICE)
    # the pool: pages dealt out in no order, a few of nobody's
    per = [-(-(n + b) // page) for n, b in seqs]
    s.pages_per_row = max(per)
    pool = sum(per) + 3
    order = torch.randperm(pool, generator=g, device=DEVICE).to(torch.int32)
    at = torch.tensor([sum(per[:i]) for i in range(len(per))], device=DEVICE).unsqueeze(1)
    i = torch.arange(s.pages_per_row, device=DEVICE).unsqueeze(0)
    gone = torch.tensor([max(0, b + 1 - case["window"]) // page if case["window"] else 0 for b in s.before], device=DEVICE).unsqueeze(1)
    held = (i < torch.tensor(per, device=DEVICE).unsqueeze(1)) & (i >= gone)
    s.page_table = torch.where(held, order[(at + i).clamp(max=pool - 1)], -1).to(torch.int32).contiguous()
    kind = torch.float8_e4m3fn if case["e4m3"] else torch.bfloat16
    s.k_scale, s.v_scale = (K_SCALE, V_SCALE) if case["e4m3"] else (1.0, 1.0)
    fill = lambda scale: (torch.randn(pool, kv_heads, page * d, generator=g, device=DEVICE) / scale).clamp(-448, 448).to(kind)  # noqa: E731
    s.k_pages, s.v_pages = fill(s.k_scale), fill(s.v_scale)
    # cosines and sines of every position that the pages can hold
    angle = torch.arange(s.pages_per_row * page, dtype=torch.float64, device=DEVICE).unsqueeze(1) * (
        base ** (-torch.arange(0, d, 2, dtype=torch.float64, device=DEVICE) / d))
    s.rope = torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()
    seq = torch.repeat_interleave(torch.arange(len(seqs)), torch.tensor(s.new)).to(DEVICE)
    s.token_seq = seq
    s.token_pos = torch.arange(tokens, device=DEVICE) - torch.tensor(s.q_start[:-1], device=DEVICE)[seq] + torch.tensor(s.before, device=DEVICE)[seq]
    n = seqs[0][1] + 1
    s.read = torch.empty(2, n, kv_heads, d, dtype=torch.bfloat16, device=DEVICE) if case["op"] == "read" else None
    s.handle = _handle(s) if own else None
    torch.cuda.synchronize()
    return s


def _handle(s):
    """What a program keeps: the pool's description, the batch (made once per step, for all layers) and the workspace."""
    from paper_2412_17246_amd import Batch, PagedKv, load_library, op_paged_attention_workspace_bytes

    kv = PagedKv(s.page, s.kv_heads, s.d, k=s.k_pages, v=s.v_pages, page_table=s.page_table, k_scale=s.k_scale, v_scale=s.v_scale)
    batch = Batch(load_library(), s.q_start, list(range(len(s.seqs))), s.before)
    need = op_paged_attention_workspace_bytes(batch, kv, s.heads, window=s.window)
    return SimpleNamespace(kv=kv, batch=batch, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device=DEVICE))


def run(s):
    op = s.case["op"]
    if own:
        from paper_2412_17246_amd import op_paged_append, op_paged_attention, op_paged_read

        h = s.handle
        if op == "append":
            op_paged_append(h.batch, h.kv, s.k, s.v, rope=s.rope)
            return [s.k_pages, s.v_pages]
        if op == "attention":
            op_paged_attention(h.batch, h.kv, s.q, s.out, rope=s.rope, window=s.window, workspace=h.workspace)
            return s.out
        op_paged_read(h.kv, 0, 0, s.read.shape[1], s.read[0], s.read[1])
        return s.read
    if op == "append":
        return _append(s)
    if op == "attention":
        several = [i for i, n in enumerate(s.new) if n > 1]
        single = [i for i, n in enumerate(s.new) if n == 1]
        if several:
            _attend(s, several)
        if single:
            _attend(s, single)
        return s.out
    k, v = _gather(s, [0], s.read.shape[1])
    s.read.copy_(torch.stack([k[0], v[0]]).transpose(1, 2))
    return s.read


def _rotate(s, x, pos):
    """x [..., heads, d] of tokens at positions pos [...]: pairs (j, j + d/2) turned by the position's angles."""
    c, sn = s.rope[pos][..., None, :, 0], s.rope[pos][..., None, :, 1]
    lo, hi = x.float().chunk(2, dim=-1)
    return torch.cat([lo * c - hi * sn, hi * c + lo * sn], dim=-1)


def _append(s):
    tokens, d = s.qkv.shape[0], s.d
    pages = s.page_table[s.token_seq, s.token_pos // s.page].long()
    block, p = s.token_pos % s.page // 32, s.token_pos % 32
    k = _rotate(s, s.k.reshape(tokens, s.kv_heads, d), s.token_pos) / s.k_scale
    v = s.v.reshape(tokens, s.kv_heads, d).float() / s.v_scale
    kind = s.k_pages.dtype
    piece = 16 if s.case["e4m3"] else 8
    bits = torch.uint8 if s.case["e4m3"] else torch.int16
    if s.case["e4m3"]:
        k, v = k.clamp(-448, 448), v.clamp(-448, 448)
    k, v = k.to(kind).view(bits), v.to(kind).view(bits)
    there = pages >= 0
    pages, block, p, k, v = pages[there], block[there], p[there], k[there], v[there]
    heads = torch.arange(s.kv_heads, device=DEVICE)
    kp = s.k_pages.view(bits).view(-1, s.kv_heads, s.page // 32, d // piece, 32, piece)
    kp[pages[:, None], heads[None], block[:, None], :, p[:, None], :] = k.view(-1, s.kv_heads, d // piece, piece)
    t, a, h, b = p // 16, p // 8 % 2, p // 4 % 2, p % 4
    vp = s.v_pages.view(bits)
    if s.case["e4m3"]:
        vp = vp.view(-1, s.kv_heads, s.page // 32, 2, d, 16)
        vp[pages[:, None], heads[None], block[:, None], h[:, None], :, (8 * t + 4 * a + b)[:, None]] = v
    else:
        vp = vp.view(-1, s.kv_heads, s.page // 32, 4, d, 8)
        vp[pages[:, None], heads[None], block[:, None], (2 * t + h)[:, None], :, (4 * a + b)[:, None]] = v
    return [s.k_pages, s.v_pages]


def _gather(s, rows, length):
    """Keys and values [rows, kv heads, positions, d] of the first `length` positions (whole pages, cut)."""
    n, d, nb = -(-length // s.page), s.d, s.page // 32
    table = s.page_table[rows, :n].long().clamp(min=0)
    piece = 16 if s.case["e4m3"] else 8
    k = s.k_pages.view(-1, s.kv_heads, nb, d // piece, 32, piece)[table].float() * s.k_scale
    k = k.permute(0, 2, 1, 3, 5, 4, 6).reshape(len(rows), s.kv_heads, n * s.page, d)
    if s.case["e4m3"]:                                       # [rows, pages, heads, blocks, h, j, t, a, b]
        v = s.v_pages.view(-1, s.kv_heads, nb, 2, d, 2, 2, 4)[table].float() * s.v_scale
        v = v.permute(0, 2, 1, 3, 6, 7, 4, 8, 5)
    else:                                                    # [rows, pages, heads, blocks, t, h, j, a, b]
        v = s.v_pages.view(-1, s.kv_heads, nb, 2, 2, d, 2, 4)[table].float() * s.v_scale
        v = v.permute(0, 2, 1, 3, 4, 7, 5, 8, 6)
    v = v.reshape(len(rows), s.kv_heads, n * s.page, d)
    return k[:, :, :length], v[:, :, :length]


def _attend(s, rows):
    """Attention of the sequences `rows`, laid out [sequence, token] with room for the longest."""
    d, kv_heads, group = s.d, s.kv_heads, s.heads // s.kv_heads
    new = torch.tensor([s.new[r] for r in rows], device=DEVICE)
    first = torch.tensor([s.q_start[r] for r in rows], device=DEVICE)
    before = torch.tensor([s.before[r] for r in rows], device=DEVICE)
    most, length = max(s.new[r] for r in rows), max(s.new[r] + s.before[r] for r in rows)
    i = torch.arange(most, device=DEVICE)
    real = i[None] < new[:, None]
    token = (first[:, None] + i[None].minimum(new[:, None] - 1))
    pos = before[:, None] + i[None].minimum(new[:, None] - 1)
    q = _rotate(s, s.q[token.flatten()].view(len(rows), most, s.heads, d), pos) / math.sqrt(d)
    q = q.view(len(rows), most, kv_heads, group, d).permute(0, 2, 3, 1, 4).reshape(len(rows), kv_heads, group * most, d)
    k, v = _gather(s, rows, length)
    scores = (q @ k.transpose(2, 3).contiguous()).view(len(rows), kv_heads, group, most, length)
    j = torch.arange(length, device=DEVICE)
    seen = (j <= pos[..., None]) & (s.page_table[rows][:, j // s.page] >= 0)[:, None]
    if s.window:
        seen &= j > pos[..., None] - s.window
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    scores -= scores.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    scores.exp_()
    total = scores.sum(dim=-1, keepdim=True)
    o = (scores.view(len(rows), kv_heads, group * most, length) @ v).view(len(rows), kv_heads, group, most, d)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(len(rows), most, s.heads * d)
    s.out[token[real]] = o[real].to(s.out.dtype)


def work(case):
    heads, kv_heads, d, _ = SHAPES[case["shape"]]
    seqs = _lengths(case)
    item = 1 if case["e4m3"] else 2
    tokens = sum(n for n, _ in seqs)
    if case["op"] == "append":                               # rows in, positions out, cosines and sines
        return {"bytes": tokens * kv_heads * d * 2 * (2 + item) + tokens * d * 4, "flops": 3 * tokens * kv_heads * d}
    if case["op"] == "read":
        return {"bytes": (seqs[0][1] + 1) * kv_heads * d * 2 * (2 + item), "flops": 0}
    window, cached, pairs = case["window"], 0, 0
    for n, before in seqs:
        cached += min(n + before, window + n - 1) if window else n + before
        pairs += sum(min(before + i + 1, window) if window else before + i + 1 for i in range(n))
    return {"bytes": cached * kv_heads * d * 2 * item + tokens * heads * d * 2 * 2 + tokens * d * 4, "flops": 4 * heads * d * pairs}


def exact(case, seed):
    """The same from the definition in 64 bits, sequence by sequence and head by head, element offsets written out."""
    s = prepare(case, seed)
    d, page, size = s.d, s.page, s.page * s.d

    def offsets(pos):
        """Where the elements of positions `pos` of a (page, head) lie: of keys and of values, [positions, d]."""
        p, j = (pos % 32).unsqueeze(1), torch.arange(d, device=DEVICE).unsqueeze(0)
        block = (pos % page // 32).unsqueeze(1) * (32 * d)
        lane, step = (p // 4) % 2, p // 16
        e = p % 4 + 4 * (p // 8 % 2)
        if case["e4m3"]:
            return block + (j // 16 * 32 + p) * 16 + j % 16, block + (lane * d + j) * 16 + 8 * step + e
        return block + (j // 8 * 32 + p) * 8 + j % 8, block + ((2 * step + lane) * d + j) * 8 + e

    def turned(x, pos):
        theta = s.base ** (torch.arange(d // 2, dtype=torch.float64, device=DEVICE) * (-2.0 / d))
        a = pos.double().unsqueeze(-1) * theta
        z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * torch.complex(a.cos(), a.sin())
        return torch.cat([z.real, z.imag], dim=-1)

    if case["op"] == "append":
        out = [s.k_pages.double().view(-1, s.kv_heads, size), s.v_pages.double().view(-1, s.kv_heads, size)]
        for r, (n, before) in enumerate(s.seqs):
            pos = torch.arange(before, before + n, device=DEVICE)
            ko, vo = offsets(pos)
            pages = s.page_table[r, pos // page].long().unsqueeze(1)
            rows = slice(s.q_start[r], s.q_start[r + 1])
            for h in range(s.kv_heads):
                out[0][pages, h, ko] = (turned(s.k[rows, h * d:(h + 1) * d], pos) / s.k_scale).clamp(-448 if case["e4m3"] else -math.inf, 448 if case["e4m3"] else math.inf)
                out[1][pages, h, vo] = (s.v[rows, h * d:(h + 1) * d].double() / s.v_scale).clamp(-448 if case["e4m3"] else -math.inf, 448 if case["e4m3"] else math.inf)
        return [o.view(s.k_pages.shape) for o in out]
    kc, vc = s.k_pages.view(-1, s.kv_heads, size), s.v_pages.view(-1, s.kv_heads, size)

    def cached(r, h, pos):
        ko, vo = offsets(pos)
        pages = s.page_table[r, pos // page].long().unsqueeze(1)
        flat = (pages * s.kv_heads + h) * size
        bits = torch.uint8 if case["e4m3"] else torch.int16
        take = lambda c, o: c.reshape(-1).view(bits)[flat + o].view(c.dtype).double()  # noqa: E731
        return take(kc, ko) * s.k_scale, take(vc, vo) * s.v_scale

    if case["op"] == "read":
        pos = torch.arange(s.read.shape[1], device=DEVICE)
        heads = [cached(0, h, pos) for h in range(s.kv_heads)]
        return torch.stack([torch.stack([k for k, _ in heads], dim=1), torch.stack([v for _, v in heads], dim=1)])
    group = s.heads // s.kv_heads
    out = torch.zeros(s.q_start[-1], s.heads, d, dtype=torch.float64, device=DEVICE)
    for r, (n, before) in enumerate(s.seqs):
        pos = torch.arange(before, before + n, device=DEVICE)
        keys = torch.arange(max(0, before + 1 - s.window) if s.window else 0, before + n, device=DEVICE)
        keys = keys[s.page_table[r, keys // page] >= 0]
        hidden = keys > pos.unsqueeze(1)
        if s.window:
            hidden |= keys <= pos.unsqueeze(1) - s.window
        for h in range(s.kv_heads):
            k, v = cached(r, h, keys)
            for x in range(h * group, (h + 1) * group):
                q = turned(s.q[s.q_start[r]:s.q_start[r + 1], x * d:(x + 1) * d], pos)
                weights = torch.softmax((q @ k.T.contiguous() * d ** -0.5).masked_fill(hidden, -math.inf), dim=1)
                out[s.q_start[r]:s.q_start[r + 1], x] = weights @ v
    return out.view(-1, s.heads * d)
