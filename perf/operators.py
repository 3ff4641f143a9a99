"""Operators for programs that run a model's layers themselves and keep its keys and values in pages: cases as such a
program runs them.

* ``append``: a batch of ragged runs of new tokens: queries and keys normalised per head (where the model does that) and
  rotated to their positions, keys and values written to the sequences' pages (``ppd_paged_append``).
* ``attention``: the new tokens' attention over their sequences' pages, causal among the new ones (``ppd_paged_attention``).
* ``verify``: drafted tokens against the target model's logits, from given random numbers (``ppd_verify_drafts``).

A batch is ``q_start`` (the first row of every sequence, and the number of rows), ``kv_len`` (a sequence's length with its
new tokens) and a table of pages; a sequence's new tokens are its last ones.
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS, THETA = 1e-5, 10000.0


# ------------------------------------------------------------------ cases
def _batch(op, dtype, heads, kv_heads, head_dim, seqs, new, ctx, page, shape_seed, **more):
    """new, ctx: the shortest and the longest run of new tokens, and of what was there before."""
    return dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, seqs=seqs, new_min=new[0], new_max=new[1], ctx_min=ctx[0],
                ctx_max=ctx[1], page=page, shape_seed=shape_seed, **more)


def _append(*a, rope=True, norm=False):
    return _batch("append", *a, rope=rope, norm=norm)


def _attention(*a, window=0, lse=False):
    return _batch("attention", *a, window=window, lse=lse)


def _verify(dtype, vocab, seqs, drafts, shape_seed, draft_logits=True, greedy=0.0, kept=0):
    """drafts: the fewest and the most of a sequence; greedy: the share of sequences that decode by arg max; kept: tokens of a
    row that top-k filtering has left above minus infinity (0: all)."""
    return dict(op="verify", dtype=dtype, vocab=vocab, seqs=seqs, draft_min=drafts[0], draft_max=drafts[1], shape_seed=shape_seed,
                draft_logits=draft_logits, greedy=greedy, kept=kept)


def listed():
    cases = {
        # one token of one conversation, heads of the 7B shape: latency
        "append_token": _append("bf16", 32, 32, 128, 1, (1, 1), (700, 700), 16, 1),
        # a server's step of drafted tokens: shared heads, heads normalised, conversations of any length up to 100k tokens
        "append_drafts_far": _append("bf16", 32, 8, 128, 24, (1, 8), (200, 100000), 16, 2, norm=True),
        # prompts of the OPT-125m shape with its fp32 cache: learned positions, nothing but the copy into pages
        "append_prompts_fp32": _append("fp32", 12, 12, 64, 5, (60, 300), (0, 0), 32, 3, rope=False),
        # long prompts of the 13B shape together
        "append_prompts": _append("bf16", 40, 40, 128, 3, (1200, 3000), (0, 0), 16, 4),
        # one token of one conversation, heads of the 7B shape: latency
        "attention_token": _attention("bf16", 32, 32, 128, 1, (1, 1), (700, 700), 16, 5),
        # k = 3 drafts behind the last token, fp32 cache of the OPT-125m shape
        "attention_drafts_fp32": _attention("fp32", 12, 12, 64, 6, (4, 4), (100, 1900), 16, 6),
        # a server's decode batch: shared heads, lengths that differ a hundredfold
        "attention_batch": _attention("bf16", 32, 8, 128, 64, (1, 1), (60, 8000), 16, 7),
        # a chunk of a long document on top of what was there, 13B heads, fp16; the log sums for a merge with another part
        "attention_chunk": _attention("fp16", 40, 40, 128, 1, (500, 500), (4000, 4000), 64, 8, lse=True),
        # whole prompts, compute-bound
        "attention_prompts": _attention("bf16", 32, 8, 128, 2, (3700, 4096), (0, 0), 16, 9),
        # one conversation by arg max, k = 3 drafts
        "verify_greedy": _verify("fp32", 32000, 1, (3, 3), 10, draft_logits=False, greedy=1.0),
        # a server's step: sampled and greedy conversations, the drafter's distributions at hand
        "verify_batch": _verify("fp32", 50272, 24, (1, 6), 11, greedy=0.25),
        # the largest: many conversations, bf16 logits, long drafts
        "verify_large": _verify("bf16", 32000, 128, (4, 8), 12),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lengths(c):
    """(new tokens, length with them) of every sequence."""
    rng = random.Random(c["shape_seed"])
    new = [rng.randint(c["new_min"], c["new_max"]) for _ in range(c["seqs"])]
    ctx = [_log_int(rng, c["ctx_min"], c["ctx_max"]) if c["ctx_min"] else c["ctx_max"] for _ in range(c["seqs"])]
    return new, [n + x for n, x in zip(new, ctx)]


def _drafts(c):
    rng = random.Random(c["shape_seed"])
    return [rng.randint(c["draft_min"], c["draft_max"]) for _ in range(c["seqs"])]


def _small_enough(c):
    """No larger than the largest listed cases of its kind, padded to its longest sequence neither."""
    w, listed_ones = work(c), [work(x) for x in listed() if x["op"] == c["op"]]
    if any(w[k] > max(x[k] for x in listed_ones) for k in w):
        return False
    if c["op"] == "verify":
        return True
    new, kv = _lengths(c)
    if c["op"] == "append":
        return c["seqs"] * max(kv) <= 1 << 22
    return c["seqs"] * c["heads"] * max(new) * max(kv) <= 1 << 30 and c["seqs"] * max(kv) * c["kv_heads"] * c["head_dim"] <= 1 << 29


def _draw_one(rng):
    op = rng.choice(["append", "attention", "attention", "verify"])
    seed = rng.randint(100, 10 ** 6)
    if op == "verify":
        lo = rng.randint(0, 8)
        return _verify(rng.choice(["fp32", "fp32", "bf16", "fp16"]), _log_int(rng, 600, 130000), _log_int(rng, 1, 128), (lo, rng.randint(lo, 10)), seed,
                       draft_logits=rng.random() < 0.7, greedy=rng.choice([0.0, 0.0, 0.3, 1.0]), kept=rng.choice([0, 0, 50]))
    kv_heads = rng.choice([1, 2, 4, 8, 8, 12, 32, 40])
    heads = kv_heads * (rng.choice([1, 2, 3, 4, 5, 7, 8, 16]) if kv_heads < 12 else 1)
    seqs = _log_int(rng, 1, 96)
    lo = rng.choice([1, 1, _log_int(rng, 1, 4000)])
    new = (lo, lo if rng.random() < 0.4 else _log_int(rng, lo, 4096))
    lo = rng.choice([0, _log_int(rng, 1, 30000)])
    ctx = (lo, lo if rng.random() < 0.4 or not lo else _log_int(rng, lo, 32000))
    shape = (rng.choice(["bf16", "bf16", "fp16", "fp32"]), heads, kv_heads, rng.choice([64, 128, 128]), seqs, new, ctx, rng.choice([8, 16, 16, 20, 32, 64, 128]), seed)
    if op == "append":
        return _append(*shape, rope=rng.random() < 0.8, norm=rng.random() < 0.5)
    return _attention(*shape, window=_log_int(rng, 30, 5000) if rng.random() < 0.25 else 0, lse=rng.random() < 0.3)


def draw(rng):
    while True:
        c = _draw_one(rng)
        if _small_enough(c):
            return c


# ------------------------------------------------------------------ inputs
def _tokens(c, seed):
    """A batch of new tokens with its pages: everything both operators on a cache share."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, hd, page = DTYPES[c["dtype"]], c["head_dim"], c["page"]
    new, kv = _lengths(c)
    n = sum(new)
    # which pages a call may touch: those of the new tokens for an append, those within the window for attention
    first = [x - m if c["op"] == "append" else max(0, x - m - c["window"] + 1) if c["window"] else 0 for m, x in zip(new, kv)]
    per_seq = max(-(-x // page) for x in kv)
    rows = np.full((c["seqs"], per_seq), -1, dtype=np.int32)      # -1: no page (not used here any more, or held elsewhere)
    used = [(s, p) for s in range(c["seqs"]) for p in range(first[s] // page, -(-kv[s] // page))]
    order = np.random.default_rng(seed).permutation(len(used))
    for (s, p), i in zip(used, order):
        rows[s, p] = i

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dt)

    s = SimpleNamespace(op=c["op"], seqs=c["seqs"], n=n, heads=c["heads"], kv_heads=c["kv_heads"], hd=hd, page=page, dtype=dt, most_new=max(new), most_kv=max(kv))
    s.q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    s.kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s.pages = torch.from_numpy(rows).cuda()
    s.k_cache = normal(max(1, len(used)), page, c["kv_heads"], hd)
    s.v_cache = normal(max(1, len(used)), page, c["kv_heads"], hd)
    # queries and keys as they come out of one projection: heads' rows of q, k and v side by side
    both = normal(n, c["heads"] + 2 * c["kv_heads"], hd)
    s.q, s.k, s.v = both[:, :c["heads"]], both[:, c["heads"]:c["heads"] + c["kv_heads"]], both[:, c["heads"] + c["kv_heads"]:]
    return s, g


def _logits(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    drafts = _drafts(c)
    n = sum(drafts) + c["seqs"]
    dt, v = DTYPES[c["dtype"]], c["vocab"]
    s = SimpleNamespace(op="verify", seqs=c["seqs"], n=n, vocab=v)
    z = torch.randn((n, v), generator=g, device="cuda").mul_(3.0)
    zd = z + torch.randn((n, v), generator=g, device="cuda").mul_(0.8)
    if c["kept"]:
        for x in (z, zd):
            x.masked_fill_(x < torch.topk(x, min(c["kept"], v), dim=1).values[:, -1:], -math.inf)
    s.target = z.to(dt)
    zd = zd.to(dt)
    s.row_start = torch.tensor(np.concatenate([[0], np.cumsum([d + 1 for d in drafts])]), dtype=torch.int32, device="cuda")
    rng = random.Random(c["shape_seed"] + 1)
    temps = [0.0 if rng.random() < c["greedy"] else rng.uniform(0.5, 1.2) for _ in range(c["seqs"])]
    s.temperature = torch.tensor(temps, dtype=torch.float32, device="cuda")
    per_row = torch.repeat_interleave(s.temperature, torch.tensor([d + 1 for d in drafts], device="cuda"))[:, None]
    # the drafter's choice: drawn from its distribution, or its most probable token
    noise = -torch.log(-torch.log(torch.rand((n, v), generator=g, device="cuda").clamp_(1e-9, 1 - 1e-6)))
    noise = noise * per_row if c["draft_logits"] else torch.zeros_like(noise)
    drawn = torch.argmax(zd.float() + noise, dim=1).to(torch.int32)
    s.ids = torch.cat([torch.randint(0, v, (1,), generator=g, device="cuda", dtype=torch.int32), drawn[:-1]])      # row r + 1 is what row r's drafter drew
    s.draft = zd if c["draft_logits"] else None
    s.uniform = torch.rand((n, 2), generator=g, device="cuda")
    return s


def prepare(case, seed):
    c = case
    if c["op"] == "verify":
        return _logits(c, seed)
    s, g = _tokens(c, seed)
    if c["op"] == "append":
        s.rotary = s.hd if c["rope"] else 0
        s.q_gain, s.k_gain = ((1 + 0.1 * torch.randn((2, s.hd), generator=g, device="cuda")).to(s.dtype) if c["norm"] else (None, None))
    else:
        s.q = s.q.contiguous()
        s.window, s.lse = c["window"], c["lse"]
    return s


# ------------------------------------------------------------------ one pass
def _own():
    from paper_2307_05908_amd import binding      # only where `own` is set, which happens after this file has been read
    return binding


def run(state):
    s = state
    if s.op == "append":
        if own:
            q = _own().ppd_paged_append(s.k_cache, s.v_cache, s.pages, s.q_start, s.kv_len, s.q, s.k, s.v, q_gain=s.q_gain, k_gain=s.k_gain, norm_eps=EPS,
                                        rotary_dim=s.rotary, rope_theta=THETA)
        else:
            q = _append_plain(s)
        return {"q": q, "k_cache": s.k_cache, "v_cache": s.v_cache}
    if s.op == "attention":
        if own:
            out, lse = _own().ppd_paged_attention(s.q, s.k_cache, s.v_cache, s.pages, s.q_start, s.kv_len, window=s.window, want_lse=s.lse)
        else:
            out, lse = _attention_plain(s)
        return {"out": out, "lse": lse} if s.lse else {"out": out}
    if own:
        tokens, accepted = _own().ppd_verify_drafts(s.target, s.ids, s.row_start, s.uniform, draft_logits=s.draft, temperature=s.temperature)
    else:
        tokens, accepted = _verify_plain(s)
    return {"tokens": tokens, "accepted": accepted}


def _rows_of(start, n):
    """Every row's sequence, and its place there."""
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(start, row, right=True) - 1
    return seq, row - start[seq]


def _append_plain(s):
    seq, i = _rows_of(s.q_start, s.n)
    pos = (s.kv_len[seq] - (s.q_start[seq + 1] - s.q_start[seq]) + i).long()

    def head_norm(x, gain):
        x = x.float()
        return x if gain is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()

    def rotate(x):
        if not s.rotary:
            return x
        half = s.rotary // 2
        angle = pos.double()[:, None] * THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        lo, hi, rest = x[..., :half], x[..., half:s.rotary], x[..., s.rotary:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, rest], -1)

    page, at = s.pages[seq, pos // s.page].long(), pos % s.page
    s.k_cache[page, at] = rotate(head_norm(s.k, s.k_gain)).to(s.dtype)
    s.v_cache[page, at] = s.v
    return rotate(head_norm(s.q, s.q_gain)).to(s.dtype)


def _attention_plain(s):
    """Padded to the longest run and the longest sequence."""
    group, nm, km = s.heads // s.kv_heads, s.most_new, s.most_kv
    seq, i = _rows_of(s.q_start, s.n)
    count = s.q_start[1:] - s.q_start[:-1]
    row = (s.q_start[:-1, None] + torch.arange(nm, device="cuda")).clamp(max=s.n - 1)
    q = s.q[row].float().view(s.seqs, nm, s.kv_heads, group, s.hd).permute(0, 2, 3, 1, 4).reshape(s.seqs, s.kv_heads, group * nm, s.hd)
    pos = torch.arange(km, device="cuda")
    page = s.pages[:, pos // s.page].long()
    k = s.k_cache[page.clamp(min=0), pos % s.page].float().permute(0, 2, 3, 1).contiguous()
    score = torch.matmul(q, k).mul_(1 / math.sqrt(s.hd)).view(s.seqs, s.kv_heads, group, nm, km)
    at = ((s.kv_len - count)[:, None] + torch.arange(nm, device="cuda"))[:, :, None]
    seen = (pos <= at) & (page >= 0)[:, None]
    if s.window:
        seen &= pos > at - s.window
    score.masked_fill_(~seen[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    most = torch.where(torch.isinf(most), torch.zeros_like(most), most)
    weight = score.sub_(most).exp_()
    total = weight.sum(-1, keepdim=True)
    v = s.v_cache[page.clamp(min=0), pos % s.page].float().permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(weight.view(s.seqs, s.kv_heads, group * nm, km), v).view(s.seqs, s.kv_heads, group, nm, s.hd) / torch.where(total > 0, total, torch.ones_like(total))
    out = out.permute(0, 3, 1, 2, 4).reshape(s.seqs, nm, s.heads, s.hd)[seq, i].to(s.dtype)
    lse = (most + torch.log(total)).permute(0, 3, 1, 2, 4).reshape(s.seqs, nm, s.heads)[seq, i] if s.lse else None
    return out, lse


def _verify_plain(s):
    """In 64 bits: which token a random number falls on is a matter of the last digits of long sums."""
    seq, _ = _rows_of(s.row_start, s.n)
    row = torch.arange(s.n, device="cuda")
    last = row + 1 == s.row_start[seq + 1]
    temp = s.temperature[seq].double()[:, None]
    by_max = temp <= 0

    def probabilities(z):
        z = z.double()
        e = torch.exp((z - z.amax(-1, keepdim=True)) / torch.where(by_max, torch.ones_like(temp), temp))
        return e / e.sum(-1, keepdim=True)

    best = torch.argmax(s.target, dim=-1)
    p = probabilities(s.target)
    d = s.ids[(row + 1).clamp(max=s.n - 1)].long()[:, None]
    q = probabilities(s.draft) if s.draft is not None else torch.zeros_like(p).scatter_(1, d, 1.0)
    u = s.uniform.double()
    ok = torch.where(by_max[:, 0], best == d[:, 0], u[:, 0] * q.gather(1, d)[:, 0] < p.gather(1, d)[:, 0]) & ~last
    # a sequence ends at its first row that does not take its draft
    end = torch.full((s.seqs,), s.n, device="cuda").scatter_reduce(0, seq, torch.where(ok, s.n, row), "amin")
    p, q = p[end], q[end]
    left = torch.where(last[end][:, None], p, (p - q).clamp(min=0))
    left = torch.where(left.sum(-1, keepdim=True) > 0, left, p)
    upto = torch.cumsum(left, -1)
    drawn = (upto <= u[end, 1:] * upto[:, -1:]).sum(-1).clamp(max=s.vocab - 1)
    drawn = torch.where(by_max[end, 0], best[end], drawn).to(torch.int32)
    tokens = torch.where(row < end[seq], d[:, 0].to(torch.int32), torch.where(row == end[seq], drawn[seq], -1))
    return tokens, (end - s.row_start[:-1]).to(torch.int32)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "verify":
        n = sum(_drafts(c))
        values = (n + c["seqs"]) * c["vocab"] + (n * c["vocab"] if c["draft_logits"] else 0)
        return {"bytes": values * DTYPES[c["dtype"]].itemsize, "flops": 4 * values}
    new, kv = _lengths(c)
    size, hd = DTYPES[c["dtype"]].itemsize, c["head_dim"]
    if c["op"] == "append":
        values = sum(new) * (c["heads"] + 2 * c["kv_heads"]) * hd
        return {"bytes": 2 * values * size, "flops": sum(new) * (c["heads"] + c["kv_heads"]) * hd * ((3 if c["rope"] else 0) + (4 if c["norm"] else 0))}
    w = c["window"] or 1 << 40
    pairs = sum(min(x - n + i + 1, w) for n, x in zip(new, kv) for i in range(n))
    read = sum(min(x, w + n - 1) for n, x in zip(new, kv))
    return {"bytes": (2 * sum(new) * c["heads"] + 2 * read * c["kv_heads"]) * hd * size + (4 * sum(new) * c["heads"] if c["lse"] else 0),
            "flops": 4 * pairs * c["heads"] * hd}


# ------------------------------------------------------------------ the same in 64 bits
def _append_exact(s):
    f64 = torch.float64
    kc, vc = s.k_cache.to(f64), s.v_cache.to(f64)
    start, kv, pages = s.q_start.tolist(), s.kv_len.tolist(), s.pages.cpu()
    qs = []
    for b in range(s.seqs):
        m = start[b + 1] - start[b]
        p = torch.arange(kv[b] - m, kv[b])
        turned = []
        for x, gain in ((s.q, s.q_gain), (s.k, s.k_gain)):
            x = x[start[b]:start[b + 1]].to(f64)
            if gain is not None:
                x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / s.hd + EPS) * gain.to(f64)
            if s.rotary:      # pairs as complex numbers, turned
                half = s.rotary // 2
                angle = p.to("cuda", f64)[:, None] / THETA ** (torch.arange(half, device="cuda", dtype=f64) * 2 / s.rotary)
                z = torch.complex(x[..., :half].contiguous(), x[..., half:s.rotary].contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
                x = torch.cat([z.real, z.imag, x[..., s.rotary:]], -1)
            turned.append(x)
        where = pages[b][p // s.page].long().cuda(), (p % s.page).cuda()
        kc[where], vc[where] = turned[1], s.v[start[b]:start[b + 1]].to(f64)
        qs.append(turned[0])
    return {"q": torch.cat(qs), "k_cache": kc, "v_cache": vc}


def _attention_exact(s):
    f64 = torch.float64
    out = torch.zeros((s.n, s.heads, s.hd), dtype=f64, device="cuda")
    lse = torch.full((s.n, s.heads), -math.inf, dtype=f64, device="cuda")
    start, kv, pages = s.q_start.tolist(), s.kv_len.tolist(), s.pages.cpu()
    for b in range(s.seqs):
        lo, hi, m = start[b], start[b + 1], start[b + 1] - start[b]
        p = torch.arange(kv[b])
        p = p[pages[b][p // s.page] >= 0]
        where = pages[b][p // s.page].long().cuda(), (p % s.page).cuda()
        keys, values, p = s.k_cache[where].to(f64), s.v_cache[where].to(f64), p.cuda()
        mine = torch.arange(kv[b] - m, kv[b], device="cuda")[:, None]
        hidden = p[None] > mine
        if s.window:
            hidden |= mine - p[None] >= s.window
        for h in range(s.heads):
            j = h // (s.heads // s.kv_heads)
            z = s.q[lo:hi, h].to(f64) @ keys[:, j].t().contiguous() / s.hd ** 0.5
            z[hidden] = -math.inf
            lse[lo:hi, h] = torch.logsumexp(z, -1)
            some = ~hidden.all(-1)
            out[lo:hi, h][some] = torch.softmax(z[some], -1) @ values[:, j].contiguous()
    return {"out": out, "lse": lse} if s.lse else {"out": out}


def _verify_exact(s):
    start, ids, temp, u = s.row_start.tolist(), s.ids.tolist(), s.temperature.double().tolist(), s.uniform.double().cpu().numpy()
    tokens, accepted = np.full(s.n, -1, dtype=np.int32), np.zeros(s.seqs, dtype=np.int32)

    def softmax(z, t):
        z = z.double().cpu().numpy() / t
        e = np.exp(z - z.max())
        return e / e.sum()

    for b in range(s.seqs):
        for r in range(start[b], start[b + 1]):
            if temp[b] <= 0:
                choice = int(np.argmax(s.target[r].float().cpu().numpy()))
                take = r + 1 < start[b + 1] and ids[r + 1] == choice
            else:
                p = softmax(s.target[r], temp[b])
                left, take = p, False
                if r + 1 < start[b + 1]:
                    d = ids[r + 1]
                    q = softmax(s.draft[r], temp[b]) if s.draft is not None else np.eye(1, s.vocab, d)[0]
                    take = u[r, 0] * q[d] < p[d]
                    left = np.maximum(p - q, 0)
                    left = left if left.sum() > 0 else p
                if not take:
                    upto = np.cumsum(left)
                    choice = min(int(np.searchsorted(upto, u[r, 1] * upto[-1], side="right")), s.vocab - 1)
            if not take:
                tokens[r] = choice
                break
            tokens[r] = ids[r + 1]
            accepted[b] += 1
    return {"tokens": torch.from_numpy(tokens).cuda(), "accepted": torch.from_numpy(accepted).cuda()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _append_exact, "attention": _attention_exact, "verify": _verify_exact}[s.op](s)
