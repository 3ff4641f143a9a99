"""Operators around a server's step that checks drafts, for programs that keep keys and values in 4 bits: cases as such a program runs them.

* ``plan``: a step's lengths turned into row starts, pages taken and given back, positions and slots (``ppd_paged_plan``).
* ``append``: queries and keys normalised per head (where the model does that) and rotated, keys and values written to pages of 4-bit
  numbers with a scale for every 32 (``ppd_paged_append_fp4``).
* ``attention``: the new tokens' attention over such pages, causal among the new ones (``ppd_paged_attention_fp4``).
* ``adjust``: penalties for repeated tokens, biases and grammar masks on the logits of last tokens and drafts (``ppd_adjust_logits``).

A batch is ``q_start`` (the first row of every sequence, and the number of rows), ``kv_len`` (a sequence's length with its new tokens) and a
table of pages; a sequence's new tokens are its last ones.  A 4-bit number is sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3,
4, 6; a scale is a power of two, as a byte with 127 for 1; the even one of two neighbours lies in the low half of a byte.
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS, THETA = float(np.float32(1e-5)), 10000.0
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LOWEST, HIGHEST = -125, 125      # exponents of scales


# ------------------------------------------------------------------ cases
def _plan(seqs, page, ctx, drafts, admitted, prompt, ended, free, shape_seed):
    """ctx: the shortest and the longest conversation; drafts: the most of a step; admitted, ended: shares of new and of closed
    conversations; prompt: the new ones' shortest and longest; free: free pages as a share of what the step asks for."""
    return dict(op="plan", seqs=seqs, page=page, ctx_min=ctx[0], ctx_max=ctx[1], drafts=drafts, admitted=admitted, prompt_min=prompt[0], prompt_max=prompt[1],
                ended=ended, free=free, shape_seed=shape_seed)


def _batch(op, dtype, heads, kv_heads, head_dim, seqs, new, ctx, page, shape_seed, **more):
    """new, ctx: the shortest and the longest run of new tokens, and of what was there before."""
    return dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, seqs=seqs, new_min=new[0], new_max=new[1], ctx_min=ctx[0],
                ctx_max=ctx[1], page=page, shape_seed=shape_seed, **more)


def _append(*a, rope=True, norm=False):
    return _batch("append", *a, rope=rope, norm=norm)


def _attention(*a, window=0, lse=False):
    return _batch("attention", *a, window=window, lse=lse)


def _adjust(dtype, vocab, seqs, drafts, history, shape_seed, penalties=True, biases=0, masked=0.0):
    """drafts: the fewest and the most of a sequence; history: the shortest and the longest; biases: the most of a sequence; masked: the
    share of rows that a grammar binds."""
    return dict(op="adjust", dtype=dtype, vocab=vocab, seqs=seqs, draft_min=drafts[0], draft_max=drafts[1], history_min=history[0], history_max=history[1],
                penalties=penalties, biases=biases, masked=masked, shape_seed=shape_seed)


def listed():
    cases = {
        # a server's step of drafted tokens, a conversation or two that end or begin: latency
        "plan_step": _plan(24, 16, (200, 8000), 8, 0.1, (100, 600), 0.1, 2.0, 1),
        # a busy server's: thousands of conversations, prompts among them, and fewer free pages than they ask for
        "plan_admit": _plan(2048, 16, (60, 8000), 4, 0.05, (100, 4000), 0.05, 0.8, 2),
        # one token of one conversation, heads of the 7B shape: latency
        "append_token": _append("bf16", 32, 32, 128, 1, (1, 1), (700, 700), 16, 3),
        # long prompts of the 13B shape together
        "append_prompts": _append("bf16", 40, 40, 128, 3, (1200, 3000), (0, 0), 16, 4),
        # one token of one conversation, heads of the 7B shape: latency
        "attention_token": _attention("bf16", 32, 32, 128, 1, (1, 1), (700, 700), 16, 5),
        # k = 3 drafts behind the last token, fp32 rows of the OPT-125m shape
        "attention_drafts_fp32": _attention("fp32", 12, 12, 64, 6, (4, 4), (100, 1900), 16, 6),
        # a server's decode batch: shared heads, conversations long enough that 4 bits are what they fit in
        "attention_batch": _attention("bf16", 32, 8, 128, 64, (1, 1), (400, 32000), 16, 7),
        # a chunk of a long document on top of what was there, 13B heads, fp16; the log sums for a merge with another part
        "attention_chunk": _attention("fp16", 40, 40, 128, 1, (500, 500), (4000, 4000), 64, 8, lse=True),
        # whole prompts, compute-bound
        "attention_prompts": _attention("bf16", 32, 8, 128, 2, (3700, 4096), (0, 0), 16, 9),
        # one conversation, k = 3 drafts, penalties over its last 700 tokens
        "adjust_one": _adjust("fp32", 32000, 1, (3, 3), (700, 700), 10),
        # a server's step: penalties and biases, a third of the rows bound by a grammar
        "adjust_batch": _adjust("fp32", 50272, 24, (1, 6), (50, 4000), 11, biases=40, masked=0.3),
        # the largest: many conversations, bf16 logits, long drafts and histories
        "adjust_large": _adjust("bf16", 32000, 128, (4, 8), (200, 8000), 12, biases=10, masked=0.1),
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


def _requests(c):
    """(positions held, kept, and tokens wanted) of every sequence, and the free pages."""
    rng = random.Random(c["shape_seed"])
    held, kept, wanted = [], [], []
    for _ in range(c["seqs"]):
        x = rng.random()
        if x < c["admitted"]:
            held.append(0)
            kept.append(0)
            wanted.append(_log_int(rng, c["prompt_min"], c["prompt_max"]))
        else:
            held.append(_log_int(rng, c["ctx_min"], c["ctx_max"]) + 1 + c["drafts"])
            end = x < c["admitted"] + c["ended"]
            kept.append(0 if end else held[-1] - rng.randint(0, c["drafts"]))
            wanted.append(0 if end else 1 + c["drafts"])
    pages = sum(max(0, -(-(k + w) // c["page"]) - -(-h // c["page"])) for h, k, w in zip(held, kept, wanted))
    return held, kept, wanted, int(pages * c["free"])


def _rows_in(c):
    """(rows of every sequence, tokens before them)."""
    rng = random.Random(c["shape_seed"])
    rows = [1 + rng.randint(c["draft_min"], c["draft_max"]) for _ in range(c["seqs"])]
    return rows, [_log_int(rng, c["history_min"], c["history_max"]) for _ in rows]


def _small_enough(c):
    """No larger than the largest listed cases of its kind, padded to its longest sequence neither."""
    w, listed_ones = work(c), [work(x) for x in listed() if x["op"] == c["op"]]
    if any(w[k] > max(x[k] for x in listed_ones) for k in w):
        return False
    if c["op"] == "plan":
        return True
    if c["op"] == "adjust":
        return c["seqs"] * c["history_max"] <= 1 << 21
    new, kv = _lengths(c)
    if c["op"] == "append":
        return c["seqs"] * max(kv) <= 1 << 22
    return c["seqs"] * c["heads"] * max(new) * max(kv) <= 1 << 30 and c["seqs"] * max(kv) * c["kv_heads"] * c["head_dim"] <= 1 << 31


def _draw_one(rng):
    op = rng.choice(["plan", "append", "attention", "attention", "adjust"])
    seed = rng.randint(100, 10 ** 6)
    page = rng.choice([8, 16, 16, 20, 32, 64, 128])
    if op == "plan":
        lo, short = _log_int(rng, 1, 8000), _log_int(rng, 1, 4000)
        return _plan(_log_int(rng, 1, 4096), page, (lo, _log_int(rng, lo, 16000)), rng.randint(0, 10), rng.choice([0.0, 0.05, 0.5]), (short, _log_int(rng, short, 4000)),
                     rng.choice([0.0, 0.05, 0.3]), rng.choice([0.0, 0.5, 0.9, 3.0]), seed)
    if op == "adjust":
        lo, short = rng.randint(0, 8), _log_int(rng, 1, 10000)
        return _adjust(rng.choice(["fp32", "fp32", "bf16", "fp16"]), _log_int(rng, 600, 130000), _log_int(rng, 1, 128), (lo, rng.randint(lo, 10)),
                       (short, _log_int(rng, short, 30000)), seed, penalties=rng.random() < 0.8, biases=rng.choice([0, 0, 5, 300]), masked=rng.choice([0.0, 0.0, 0.2, 1.0]))
    kv_heads = rng.choice([1, 2, 4, 8, 8, 12, 32, 40])
    heads = kv_heads * (rng.choice([1, 2, 4, 5, 7, 8, 16]) if kv_heads < 12 else 1)
    seqs = _log_int(rng, 1, 96)
    lo = rng.choice([1, 1, _log_int(rng, 1, 4000)])
    new = (lo, lo if rng.random() < 0.4 else _log_int(rng, lo, 4096))
    lo = rng.choice([0, _log_int(rng, 1, 60000)])
    ctx = (lo, lo if rng.random() < 0.4 or not lo else _log_int(rng, lo, 64000))
    shape = (rng.choice(["bf16", "bf16", "fp16", "fp32"]), heads, kv_heads, rng.choice([64, 128, 128]), seqs, new, ctx, page, seed)
    if op == "append":
        return _append(*shape, rope=rng.random() < 0.8, norm=rng.random() < 0.5)
    return _attention(*shape, window=_log_int(rng, 30, 5000) if rng.random() < 0.25 else 0, lse=rng.random() < 0.3)


def draw(rng):
    while True:
        c = _draw_one(rng)
        if _small_enough(c):
            return c


# ------------------------------------------------------------------ 4-bit numbers
def _quantised(x):
    """Rows of multiples of 32 numbers as (codes, scales, the values that they stand for): the least scale that no number's rounding goes
    beyond half a step with (up to 7 counts as 6), numbers to nearest, ties to even."""
    b = x.unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(most)                                # most = part * 2^power, 0.5 <= part < 1
    e = torch.where(most > 0, power - 3 + (part > 0.875).to(power.dtype), torch.full_like(power, LOWEST)).clamp(LOWEST, HIGHEST)
    y = torch.ldexp(b, -e)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8) + (a > 2.5).to(torch.uint8) +
            (a >= 3.5).to(torch.uint8) + (a > 5).to(torch.uint8))
    value = torch.ldexp(torch.where(y < 0, -1.0, 1.0).to(x.dtype) * torch.tensor(GRID, device=x.device, dtype=x.dtype)[code.int()], e).flatten(-2)
    code = (code + 8 * (y < 0).to(torch.uint8)).flatten(-2)
    return code[..., ::2] + 16 * code[..., 1::2], (e[..., 0] + 127).to(torch.uint8), value


def _values(codes, scales):
    """The numbers that codes and scales stand for."""
    lut = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    pairs = torch.stack([lut[(codes & 15).int()], lut[(codes >> 4).int()]], -1).flatten(-2)
    return torch.ldexp(pairs.unflatten(-1, (-1, 32)), scales.int()[..., None] - 127).flatten(-2)


# ------------------------------------------------------------------ inputs
def _pool(c, seed):
    held, kept, wanted, free = _requests(c)
    page = c["page"]
    rows = [h // page + (h % page > 0) for h in held]
    wide = max(max(rows), max(-(-(k + w) // page) for k, w in zip(kept, wanted)))
    n_pages = sum(rows) + max(1, free)
    order = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.full((c["seqs"], wide), -1, dtype=np.int32)
    table[np.arange(wide)[None] < np.asarray(rows)[:, None]] = order[:sum(rows)]
    s = SimpleNamespace(op="plan", seqs=c["seqs"], page=page, n_pages=n_pages, n=sum(wanted))
    s.held, s.kept, s.wanted = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (held, kept, wanted))
    s.pages = torch.from_numpy(table).cuda()
    # the ring of free pages: pages taken and given back since it was filled, and the numbers of those that lie between
    head = seed % 1000
    ring = np.full(n_pages, -1, dtype=np.int32)
    ring[(head + np.arange(n_pages - sum(rows))) % n_pages] = order[sum(rows):]
    s.ring = torch.from_numpy(ring).cuda()
    s.counters = torch.tensor([head, head + n_pages - sum(rows)], dtype=torch.int64, device="cuda")
    return s


def _tokens(c, seed):
    """A batch of new tokens with its pages: everything both operators on a cache share."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, hd, page = DTYPES[c["dtype"]], c["head_dim"], c["page"]
    new, kv = _lengths(c)
    n = sum(new)
    # which pages a call may touch: those of the new tokens for an append, those within the window for attention
    first = [x - m if c["op"] == "append" else max(0, x - m - c["window"] + 1) if c["window"] else 0 for m, x in zip(new, kv)]
    rows = np.full((c["seqs"], max(-(-x // page) for x in kv)), -1, dtype=np.int32)      # -1: no page (not used here any more, or held elsewhere)
    used = [(s, p) for s in range(c["seqs"]) for p in range(first[s] // page, -(-kv[s] // page))]
    order = np.random.default_rng(seed).permutation(len(used))
    for (s, p), i in zip(used, order):
        rows[s, p] = i

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = SimpleNamespace(op=c["op"], seqs=c["seqs"], n=n, heads=c["heads"], kv_heads=c["kv_heads"], hd=hd, page=page, dtype=dt, most_new=max(new), most_kv=max(kv))
    s.q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    s.kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s.pages = torch.from_numpy(rows).cuda()
    shape = (max(1, len(used)), page, c["kv_heads"], hd)
    s.k_codes, s.k_scales = _quantised(normal(*shape))[:2]
    s.v_codes, s.v_scales = _quantised(normal(*shape))[:2]
    # queries and keys as they come out of one projection: heads' rows of q, k and v side by side
    both = normal(n, c["heads"] + 2 * c["kv_heads"], hd).to(dt)
    s.q, s.k, s.v = both[:, :c["heads"]], both[:, c["heads"]:c["heads"] + c["kv_heads"]], both[:, c["heads"] + c["kv_heads"]:]
    return s, g


def _logits(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, before = _rows_in(c)
    n, v, seqs = sum(rows), c["vocab"], c["seqs"]
    s = SimpleNamespace(op="adjust", seqs=seqs, n=n, vocab=v, most_rows=max(rows), most_before=max(before))
    s.logits = torch.randn((n, v), generator=g, device="cuda").mul_(3.0).to(DTYPES[c["dtype"]])
    s.out = torch.empty_like(s.logits)
    s.row_start = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")

    def words(*shape):      # a text's: few are frequent
        return (v * torch.rand(shape, generator=g, device="cuda") ** 4).to(torch.int32).clamp_(max=v - 1)

    s.ids, s.history = words(n), words(seqs, max(before))
    s.history_len = torch.tensor(before, dtype=torch.int32, device="cuda")
    s.prompt_len = s.history_len // 3
    rng = random.Random(c["shape_seed"] + 1)

    def floats(values):
        return torch.tensor(values, dtype=torch.float32, device="cuda")

    s.repetition, s.presence, s.frequency = ((floats([rng.uniform(1.0, 1.5) for _ in rows]), floats([rng.uniform(0.0, 1.0) for _ in rows]),
                                              floats([rng.uniform(0.0, 0.5) for _ in rows])) if c["penalties"] else (None, None, None))
    s.bias_start = s.bias_ids = s.bias = s.mask = s.mask_row = None
    if c["biases"]:
        many = [rng.randint(0, c["biases"]) for _ in rows]
        s.bias_start = torch.tensor(np.concatenate([[0], np.cumsum(many)]), dtype=torch.int32, device="cuda")
        s.bias_ids = torch.randint(0, v, (max(1, sum(many)),), generator=g, device="cuda", dtype=torch.int32)
        s.bias = torch.randn(max(1, sum(many)), generator=g, device="cuda").mul_(4.0)
        s.most_biases = max(many)
    if c["masked"]:
        masks = max(1, int(n * c["masked"]))
        which = np.full(n, -1, dtype=np.int32)
        which[np.random.default_rng(seed).permutation(n)[:masks]] = np.arange(masks)
        s.mask_row = torch.from_numpy(which).cuda()
        s.mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (masks, -(-v // 32)), generator=g, device="cuda", dtype=torch.int32)      # a bit a token
        s.mask &= torch.randint(-2 ** 31, 2 ** 31 - 1, s.mask.shape, generator=g, device="cuda", dtype=torch.int32)
    return s


def prepare(case, seed):
    c = case
    if c["op"] == "plan":
        return _pool(c, seed)
    if c["op"] == "adjust":
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
    if s.op == "plan":
        if own:
            p = _own().ppd_paged_plan(s.pages, s.ring, s.counters, s.held, s.wanted, s.page, s.n, kept=s.kept)
            return {"pages": s.pages, "ring": s.ring, "q_start": p.q_start, "kv_len": p.kv_len, "granted": p.granted, "counters": p.counters,
                    "row_seq": p.row_seq, "positions": p.positions, "slots": p.slots}
        return _plan_plain(s)
    if s.op == "append":
        if own:
            q, k, v = _own().ppd_paged_append_fp4(s.k_codes, s.k_scales, s.v_codes, s.v_scales, s.pages, s.q_start, s.kv_len, s.q, s.k, s.v, q_gain=s.q_gain,
                                                  k_gain=s.k_gain, norm_eps=EPS, rotary_dim=s.rotary, rope_theta=THETA, want_values=True)
        else:
            q, k, v = _append_plain(s)
        return {"q": q, "k": k, "v": v}      # keys and values as the pages have them now
    if s.op == "attention":
        if own:
            out, lse = _own().ppd_paged_attention_fp4(s.q, s.k_codes, s.k_scales, s.v_codes, s.v_scales, s.pages, s.q_start, s.kv_len, window=s.window,
                                                      want_lse=s.lse)
        else:
            out, lse = _attention_plain(s)
        return {"out": out, "lse": lse} if s.lse else {"out": out}
    if own:
        return _own().ppd_adjust_logits(s.logits, s.row_start, ids=s.ids, history=s.history, history_len=s.history_len, prompt_len=s.prompt_len,
                                        repetition=s.repetition, presence=s.presence, frequency=s.frequency, bias_start=s.bias_start, bias_ids=s.bias_ids,
                                        bias=s.bias, mask=s.mask, mask_row=s.mask_row, out=s.out)
    return _adjust_plain(s)


def _rows_of(start, n):
    """Every row's sequence, and its place there."""
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(start, row, right=True) - 1
    return seq, row - start[seq]


def _plan_plain(s):
    """Places of all sequences as one table."""
    page, wide, n_pages = s.page, s.pages.shape[1], s.n_pages
    held = s.held.long().clamp(0, wide * page)
    kept, wanted = torch.minimum(s.kept.long().clamp(min=0), held), s.wanted.long().clamp(min=0)
    have, reach = (held + page - 1) // page, (kept + wanted + page - 1) // page
    fits = reach <= wide
    ask = torch.where(fits, wanted, 0)
    fits = fits & ((ask == 0) | (torch.cumsum(ask, 0) <= s.n))
    need = torch.where(fits, (reach - have).clamp(min=0), 0)
    fits = fits & ((need == 0) | (torch.cumsum(need, 0) <= s.counters[1] - s.counters[0]))
    granted, taken = torch.where(fits, wanted, 0), torch.where(fits, need, 0)
    kv_len = kept + granted
    want = (kv_len + page - 1) // page
    place = torch.arange(wide, device="cuda")[None]
    back = (place >= want[:, None]) & (place < have[:, None]) & (s.pages >= 0) & (s.pages < n_pages)
    nth = torch.cumsum(back.flatten().long(), 0).view_as(back) - 1
    ring = torch.cat([s.ring, s.ring[:1]])                          # one place more, for what is not given back
    ring[torch.where(back, (s.counters[1] + nth) % n_pages, n_pages)] = s.pages
    source = (s.counters[0] + (torch.cumsum(taken, 0) - taken)[:, None] + place - have[:, None]) % n_pages
    s.pages.copy_(torch.where((place >= have[:, None]) & (place < want[:, None]), s.ring[source], s.pages))
    s.ring.copy_(ring[:n_pages])
    q_start = torch.cat([torch.zeros_like(granted[:1]), torch.cumsum(granted, 0)]).to(torch.int32)
    seq, i = _rows_of(q_start, s.n)
    real = seq < s.seqs
    seq = torch.where(real, seq, 0)
    pos = kept[seq] + i
    slot = s.pages[seq, torch.where(real, pos, 0) // page].long() * page + pos % page
    return {"pages": s.pages, "ring": s.ring, "q_start": q_start, "kv_len": kv_len.to(torch.int32), "granted": granted.to(torch.int32),
            "counters": s.counters + torch.stack([taken.sum(), back.sum()]), "row_seq": torch.where(real, seq, -1).to(torch.int32),
            "positions": torch.where(real, pos, -1).to(torch.int32), "slots": torch.where(real, slot, -1)}


def _append_plain(s):
    """Keys in 64 bits: which of two 4-bit numbers is the nearer one is decided next to a border."""
    seq, i = _rows_of(s.q_start, s.n)
    pos = (s.kv_len[seq] - (s.q_start[seq + 1] - s.q_start[seq]) + i).long()

    def head_norm(x, gain):
        return x if gain is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.to(x.dtype)

    def rotate(x):
        if not s.rotary:
            return x
        half = s.rotary // 2
        angle = pos.double()[:, None] * THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        cos, sin = torch.cos(angle).to(x.dtype)[:, None], torch.sin(angle).to(x.dtype)[:, None]
        lo, hi, rest = x[..., :half], x[..., half:s.rotary], x[..., s.rotary:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, rest], -1)

    page, at = s.pages[seq, pos // s.page].long(), pos % s.page
    s.k_codes[page, at], s.k_scales[page, at], k = _quantised(rotate(head_norm(s.k.double(), s.k_gain)))
    s.v_codes[page, at], s.v_scales[page, at], v = _quantised(s.v.float())
    return rotate(head_norm(s.q.float(), s.q_gain)).to(s.dtype), k.to(s.dtype), v.to(s.dtype)


def _attention_plain(s):
    """Padded to the longest run and the longest sequence."""
    group, nm, km = s.heads // s.kv_heads, s.most_new, s.most_kv
    seq, i = _rows_of(s.q_start, s.n)
    count = s.q_start[1:] - s.q_start[:-1]
    row = (s.q_start[:-1, None] + torch.arange(nm, device="cuda")).clamp(max=s.n - 1)
    q = s.q[row].float().view(s.seqs, nm, s.kv_heads, group, s.hd).permute(0, 2, 3, 1, 4).reshape(s.seqs, s.kv_heads, group * nm, s.hd)
    pos = torch.arange(km, device="cuda")
    page = s.pages[:, pos // s.page].long()
    where = page.clamp(min=0), (pos % s.page).expand_as(page)
    k = _values(s.k_codes[where], s.k_scales[where]).permute(0, 2, 3, 1).contiguous()
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
    v = _values(s.v_codes[where], s.v_scales[where]).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(weight.view(s.seqs, s.kv_heads, group * nm, km), v).view(s.seqs, s.kv_heads, group, nm, s.hd) / torch.where(total > 0, total, torch.ones_like(total))
    out = out.permute(0, 3, 1, 2, 4).reshape(s.seqs, nm, s.heads, s.hd)[seq, i].to(s.dtype)
    lse = (most + torch.log(total)).permute(0, 3, 1, 2, 4).reshape(s.seqs, nm, s.heads)[seq, i] if s.lse else None
    return out, lse


def _adjust_plain(s):
    """Counts of all tokens for every row."""
    seq, i = _rows_of(s.row_start, s.n)
    seq = seq.long()
    x = s.logits.float()
    if s.repetition is not None:
        # a sequence's own rows up to this one, from it backwards
        back = torch.arange(s.most_rows, device="cuda")[None]
        mine = s.ids[(torch.arange(s.n, device="cuda")[:, None] - back).clamp(min=0)].long()
        at = s.history_len[seq].long()[:, None] + i[:, None] - back
        place = torch.arange(s.most_before, device="cuda")[None]
        before = s.history.long()
        zero = torch.zeros((s.seqs, s.vocab), device="cuda", dtype=torch.int32)
        there = place < s.history_len[:, None]
        any_ = zero.scatter_add(1, before, there.int())[seq].scatter_add_(1, mine, (back <= i[:, None]).int())
        out_ = zero.scatter_add(1, before, (there & (place >= s.prompt_len[:, None])).int())[seq].scatter_add_(
            1, mine, ((back <= i[:, None]) & (at >= s.prompt_len[seq].long()[:, None])).int())
        r = s.repetition[seq][:, None]
        x = torch.where(any_ > 0, torch.where(x > 0, x / r, x * r), x)
        x = x - torch.where(out_ > 0, s.frequency[seq][:, None] * out_ + s.presence[seq][:, None], 0.0)
    if s.bias is not None:
        place = torch.arange(max(1, s.most_biases), device="cuda")[None]
        e = s.bias_start[:-1, None].long() + place
        listed_ = e < s.bias_start[1:, None]
        e = torch.where(listed_, e, 0)
        # which entry of the list a token has: the last one that names it
        last = torch.zeros((s.seqs, s.vocab), device="cuda", dtype=torch.long).scatter_reduce(1, s.bias_ids[e].long(), torch.where(listed_, e + 1, 0), "amax")
        x = x + torch.where(last > 0, s.bias[(last - 1).clamp(min=0)], 0.0)[seq]
    if s.mask is not None:
        t = torch.arange(s.vocab, device="cuda")
        allowed = (s.mask[s.mask_row.clamp(min=0).long()][:, t // 32] >> (t % 32)) & 1
        x = torch.where((allowed == 0) & (s.mask_row >= 0)[:, None], -math.inf, x)
    return s.out.copy_(x)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "plan":
        held, kept, wanted, free = _requests(c)
        page = c["page"]
        moves = sum(abs(-(-(k + w) // page) - -(-h // page)) for h, k, w in zip(held, kept, wanted))
        return {"bytes": 24 * c["seqs"] + 8 * moves + 16 * sum(wanted), "flops": 4 * sum(wanted) + 20 * c["seqs"]}
    if c["op"] == "adjust":
        rows, before = _rows_in(c)
        n, size = sum(rows), DTYPES[c["dtype"]].itemsize
        return {"bytes": 2 * n * c["vocab"] * size + 4 * (sum(before) + n) + int(n * c["masked"]) * c["vocab"] // 8 + 4 * c["biases"] * c["seqs"],
                "flops": n * c["vocab"] * ((6 if c["penalties"] else 0) + (1 if c["biases"] else 0) + 1)}
    new, kv = _lengths(c)
    size, hd = DTYPES[c["dtype"]].itemsize, c["head_dim"]
    packed = hd // 2 + hd // 32
    if c["op"] == "append":
        n, kvh = sum(new), c["kv_heads"]
        # rows read; queries, codes, and the values that they stand for written
        return {"bytes": n * (2 * (c["heads"] + 2 * kvh) * hd * size + 2 * kvh * packed),
                "flops": n * hd * ((c["heads"] + kvh) * ((3 if c["rope"] else 0) + (4 if c["norm"] else 0)) + 2 * kvh * 4)}
    w = c["window"] or 1 << 40
    pairs = sum(min(x - n + i + 1, w) for n, x in zip(new, kv) for i in range(n))
    read = sum(min(x, w + n - 1) for n, x in zip(new, kv))
    return {"bytes": 2 * sum(new) * c["heads"] * hd * size + 2 * read * c["kv_heads"] * packed + (4 * sum(new) * c["heads"] if c["lse"] else 0),
            "flops": 4 * pairs * c["heads"] * hd}


# ------------------------------------------------------------------ the same in 64 bits
def _plan_exact(s):
    """One sequence after the other."""
    pages, ring, (head, tail) = s.pages.cpu().numpy().copy(), s.ring.cpu().numpy().copy(), s.counters.tolist()
    was = ring.copy()
    free, asked, needed, upto = tail - head, 0, 0, 0
    start, lens, got, seqs, positions, slots = [0], [], [], [], [], []
    taken = given = 0
    for b, (h, k, w) in enumerate(zip(s.held.tolist(), s.kept.tolist(), s.wanted.tolist())):
        have, most = -(-h // s.page), pages.shape[1] * s.page
        if k + w > most:
            w = 0
        asked += w
        if asked > s.n:
            w = 0
        need = max(0, -(-(k + w) // s.page) - have)
        needed += need
        if need and needed > free:
            w = 0
        want = -(-(k + w) // s.page)
        for j in range(have, want):
            pages[b, j] = was[(head + taken) % s.n_pages]
            taken += 1
        for j in range(want, have):
            if 0 <= pages[b, j] < s.n_pages:
                ring[(tail + given) % s.n_pages] = pages[b, j]
                given += 1
        upto += w
        start.append(upto)
        lens.append(k + w)
        got.append(w)
        seqs += [b] * w
        positions += range(k, k + w)
        slots += [int(pages[b, p // s.page]) * s.page + p % s.page for p in range(k, k + w)]
    rest = [-1] * (s.n - upto)

    def ints(x, dt=torch.int32):
        return torch.from_numpy(np.asarray(x)).to("cuda", dt)

    return {"pages": ints(pages), "ring": ints(ring), "q_start": ints(start), "kv_len": ints(lens), "granted": ints(got),
            "counters": ints([head + taken, tail + given], torch.int64), "row_seq": ints(seqs + rest), "positions": ints(positions + rest),
            "slots": ints(slots + rest, torch.int64)}


def _nearest(x):
    """The values of 4-bit rows: the exponent by trial, the number by its place among the borders."""
    f64 = torch.float64
    b = x.to(f64).unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(most.clamp(min=1e-300) / 7))
    e = torch.where(7 * torch.exp2(e - 1) >= most, e - 1, e)
    e = torch.where(7 * torch.exp2(e) < most, e + 1, e).clamp(LOWEST, HIGHEST)
    grid = torch.tensor(GRID, dtype=f64, device=x.device)
    border = (grid[1:] + grid[:-1]) / 2
    y = b / torch.exp2(e)
    at = torch.searchsorted(border, y.abs().contiguous())
    tie = (at < 7) & (y.abs() == border[at.clamp(max=6)])
    at = torch.where(tie, at + at % 2, at)
    return (torch.sign(y) * grid[at] * torch.exp2(e)).flatten(-2)


def _append_exact(s):
    f64 = torch.float64
    start, kv = s.q_start.tolist(), s.kv_len.tolist()
    qs, ks = [], []
    for b in range(s.seqs):
        m = start[b + 1] - start[b]
        p = torch.arange(kv[b] - m, kv[b])
        for x, gain, to in ((s.q, s.q_gain, qs), (s.k, s.k_gain, ks)):
            x = x[start[b]:start[b + 1]].to(f64)
            if gain is not None:
                x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / s.hd + EPS) * gain.to(f64)
            if s.rotary:      # pairs as complex numbers, turned
                half = s.rotary // 2
                angle = p.to("cuda", f64)[:, None] / THETA ** (torch.arange(half, device="cuda", dtype=f64) * 2 / s.rotary)
                z = torch.complex(x[..., :half].contiguous(), x[..., half:s.rotary].contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
                x = torch.cat([z.real, z.imag, x[..., s.rotary:]], -1)
            to.append(x)
    return {"q": torch.cat(qs), "k": _nearest(torch.cat(ks)), "v": _nearest(s.v)}


def _attention_exact(s):
    f64 = torch.float64
    out = torch.zeros((s.n, s.heads, s.hd), dtype=f64, device="cuda")
    lse = torch.full((s.n, s.heads), -math.inf, dtype=f64, device="cuda")
    start, kv, pages = s.q_start.tolist(), s.kv_len.tolist(), s.pages.cpu()
    number = torch.tensor([v for g in (1, -1) for v in (0, g / 2, g, 1.5 * g, 2 * g, 3 * g, 4 * g, 6 * g)], dtype=f64, device="cuda")

    def wide(codes, scales):
        n, h, _ = codes.shape
        x = torch.empty((n, h, s.hd), dtype=f64, device="cuda")
        x[..., 0::2], x[..., 1::2] = number[(codes % 16).long()], number[(codes // 16).long()]
        return x * torch.exp2(scales.to(f64) - 127).repeat_interleave(32, -1)

    for b in range(s.seqs):
        lo, hi, m = start[b], start[b + 1], start[b + 1] - start[b]
        p = torch.arange(kv[b])
        p = p[pages[b][p // s.page] >= 0]
        where = pages[b][p // s.page].long().cuda(), (p % s.page).cuda()
        keys, values, p = wide(s.k_codes[where], s.k_scales[where]), wide(s.v_codes[where], s.v_scales[where]), p.cuda()
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


def _adjust_exact(s):
    """Row by row, from lists of tokens."""
    f64 = torch.float64
    x = s.logits.to(f64)
    start, length, prompt = s.row_start.tolist(), s.history_len.tolist(), s.prompt_len.tolist()
    for b in range(s.seqs):
        for r in range(start[b], start[b + 1]):
            row = x[r]
            if s.repetition is not None:
                text = torch.cat([s.history[b, :length[b]], s.ids[start[b]:r + 1]]).long()
                rep, pre, fre = (float(t[b]) for t in (s.repetition, s.presence, s.frequency))
                seen = torch.unique(text)
                row[seen] = torch.where(row[seen] > 0, row[seen] / rep, row[seen] * rep)
                said, times = torch.unique(text[prompt[b]:], return_counts=True)
                row[said] -= pre + fre * times
            if s.bias is not None:
                e = range(int(s.bias_start[b]), int(s.bias_start[b + 1]))
                for t, v in dict(zip(s.bias_ids[e.start:e.stop].tolist(), s.bias[e.start:e.stop].tolist())).items():
                    row[t] += v
            if s.mask is not None and int(s.mask_row[r]) >= 0:
                bits = np.unpackbits(s.mask[int(s.mask_row[r])].cpu().numpy().view(np.uint8), bitorder="little")[:s.vocab]
                row[torch.from_numpy(bits == 0).cuda()] = -math.inf
    return x


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _plan_exact, "append": _append_exact, "attention": _attention_exact, "adjust": _adjust_exact}[s.op](s)
