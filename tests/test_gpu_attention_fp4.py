"""ppd_paged_attention_fp4 against 64 bits."""
import math

import numpy as np
import pytest
import torch

from fp4_common import NAMES, Batch4, values64
from paged_common import HALF_STEP, TINY, attention64
from paper_2307_05908_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
QUERY_TERMS, WEIGHT_TERMS = {F32: 3, BF16: 1, F16: 2}, {F32: 3, BF16: 2, F16: 2}


def call(d, **kw):
    return binding.ppd_paged_attention_fp4(d.q, d.k_codes, d.k_scales, d.v_codes, d.v_scales, d.pages, d.q_start, d.kv_len, want_lse=True, **kw)


def limits(b, ref, lse, size, reach):
    """How far (out, lse) may be off.  Keys and values are exact bf16 numbers, queries exact sums of `QUERY_TERMS` of them.  A score: as many times
    head_dim products and sums in fp32, and the scale: (terms * hd + 8) half steps of the largest sum of products, the roundings of what goes into
    exp2 among them.  The sums over n positions: as many half steps for each term of a weight, 16 for exp2 and the joins.  A weight's relative
    error counts twice (numerator and denominator).  What terms leave of a weight: 2^-9 of it each.  The result is rounded to its type.  And what
    is below fp32's smallest normal number is zero: weights under 2^-126 of the row's largest (exp2's result) and what is left of terms there, so that a
    result may be off by n * 2^-126 of the largest value, which counts where the positions that the row does see have zeros there."""
    n = max(b.kv) if b.kv else 0
    w = ((QUERY_TERMS[b.dtype] * b.hd + 8) * reach + WEIGHT_TERMS[b.dtype] * n + 16) * 2.0 ** -24
    left = 2.0 ** (-9 * WEIGHT_TERMS[b.dtype])
    gone = n * 2.0 ** -126 * float(b.v_cache.nan_to_num().abs().max())
    return size * (2 * w[..., None] + left) + ref.abs() * HALF_STEP[b.dtype] * (1 + 2.0 ** -9) + TINY[b.dtype] + gone, w + lse.abs() * 2.0 ** -23


def long_runs(d):
    """The same batch with so wide a table (of no pages) that its runs, if they are long enough, go through the kernel for long runs."""
    if d.dtype == F32 or d.n * d.heads // d.kv_heads < 64 * d.pages.shape[0]:
        return None
    most = int(13e6 / (d.n * d.heads * d.page)) + 1
    if most <= d.pages.shape[1]:
        return None
    e = object.__new__(Batch4)
    e.__dict__ = dict(d.__dict__, pages=torch.cat([d.pages, torch.full((d.pages.shape[0], most - d.pages.shape[1]), -1, dtype=torch.int32, device="cuda")], 1))
    return e


def many_heads(d):
    """The same batch with its heads so many times, and so wide a table, that sequences of 17 to 64 rows go through tiles of 32, and the number of times."""
    group, some = d.heads // d.kv_heads, min(d.n, len(d.new))
    rows = d.n * group
    sixteens = -(-rows // (16 * some)) if some else 0
    if d.dtype == F32 or rows < 20 * some or sixteens not in (2, 3, 4):
        return None, 0
    times = max(1, -(-256 // ((rows // 32 + some) * d.kv_heads)))
    if times * d.heads > 1024:
        return None, 0
    # so wide a table (of no pages) that there may be more to read than caches hold
    most = max(d.pages.shape[1], int(321e6 / (some * d.page * times * d.kv_heads * d.hd * 17 / 16)) + 1)
    pages = torch.cat([d.pages, torch.full((d.pages.shape[0], most - d.pages.shape[1]), -1, dtype=torch.int32, device=d.pages.device)], 1)
    e = object.__new__(Batch4)
    e.__dict__ = dict(d.__dict__, pages=pages, heads=times * d.heads, kv_heads=times * d.kv_heads, **{n: getattr(d, n).repeat_interleave(times, 2) for n in NAMES})
    e.q = d.q.unflatten(1, (d.kv_heads, group)).repeat_interleave(times, 1).flatten(1, 2)
    return e, times


def variants(d):
    """The batch as it is and as other kernels take it, and what makes a result (of any of these) the batch's."""
    yield d, lambda x: x
    e = long_runs(d)
    if e is not None:
        yield e, lambda x: x
    e, times = many_heads(d)
    if e is not None:
        def back(x):
            y = x.unflatten(1, (d.kv_heads, times, d.heads // d.kv_heads))
            z = y[:d.rows].nan_to_num(7.0)                   # (log sums of other rows are not written)
            assert torch.equal(z, z[:, :, :1].expand_as(z))  # (every copy of a head, to the bit)
            return y[:, :, 0].flatten(1, 2)
        yield e, back


def check(b, scale=None, window=0, d=None, ref=None):
    d = b.cuda() if d is None else d
    ref = attention64(b, scale, window) if ref is None else ref
    for i, (e, back) in enumerate(variants(d)):
        got = check_one(b, scale, window, e, back, ref)
        if i == 0:
            first = got
    return first


def check_one(b, scale, window, d, back, ref):
    out, lse = call(d, scale=scale, window=window, out=torch.full_like(d.q, 7.0))
    torch.cuda.synchronize()
    o, z = back(out).cpu().double(), back(lse).cpu().double()
    ref64, lse64, size, reach = ref
    r = b.rows
    tol, ltol = limits(b, ref64, lse64, size, reach)
    gone = torch.isinf(lse64[:r])
    assert torch.equal(torch.isinf(z[:r]) & (z[:r] < 0), gone)
    assert (o[:r][gone] == 0).all()
    assert ((z[:r] - lse64[:r]).abs()[~gone] <= ltol[:r][~gone]).all(), float((z[:r] - lse64[:r]).abs()[~gone].max())
    bad = (o[:r] - ref64[:r]).abs() > tol[:r]
    assert not bad.any() and not o[:r].isnan().any(), (bad.nonzero()[:5], o[:r][bad][:5], ref64[:r][bad][:5])
    assert (o[r:] == 7.0).all()                                        # rows of no sequence
    return out, lse


SHAPES = {
    "one": ([1], [1]),
    "token": ([1], [333]),
    "tokens": ([1, 1, 1, 0, 1], [1, 64, 65, 30, 700]),
    "drafts": ([4, 3, 1, 5], [4, 130, 17, 64]),
    "runs": ([16, 17, 0, 33, 2], [16, 80, 5, 33, 300]),
    "chunk": ([130, 1], [257, 90]),
    "prompt": ([200], [200]),
    "prompts": ([300, 250], [300, 400]),
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (6, 2), (8, 1)])
def test_types_heads_and_lengths(dtype, hd, shape, heads, kv_heads):
    new, kv = SHAPES[shape]
    check(Batch4(new, kv, heads, kv_heads, hd, dtype, seed=len(shape), pad=2))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (5, 5), (16, 1), (32, 2), (21, 3), (40, 4), (70, 2)])
def test_shared_heads(dtype, heads, kv_heads):
    check(Batch4([1, 3, 11], [50, 70, 140], heads, kv_heads, 64, dtype, seed=heads))


@pytest.mark.parametrize("page", [1, 3, 8, 16, 20, 64, 100, 256])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages(page, dtype):
    check(Batch4([1, 40, 3], [90, 130, 200], 4, 2, 128, dtype, page=page, seed=page))


@pytest.mark.parametrize("page", [1, 3, 8, 16, 20, 48, 64, 100, 256])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_pages_of_long_runs(page, dtype):
    check(Batch4([100, 1, 70], [260, 5, 90], 8, 2, 128, dtype, page=page, seed=page))
    check(Batch4([100, 1, 70], [260, 5, 90], 9, 1, 64, dtype, page=page, seed=page), window=77)


@pytest.mark.parametrize("layout,scale_layout", [("phkd", "pkhd"), ("pkhd", "phkd"), ("hpkd", "pkhd"), ("khpd", "khpd")])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 128])
def test_orders_of_the_cache(layout, scale_layout, dtype, hd):
    check(Batch4([1, 40, 3], [90, 130, 200], 4, 2, hd, dtype, layout=layout, scale_layout=scale_layout))
    if dtype == BF16:
        check(Batch4([550, 500], [570, 700], 8, 4, hd, dtype, layout=layout, scale_layout=scale_layout))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 100, 1000])
@pytest.mark.parametrize("heads", [4, 8])
def test_windows(dtype, window, heads):
    b = Batch4([1, 40, 3, 150], [190, 130, 200, 333], heads, 2, 64, dtype, seed=window)
    check(b, window=window)
    # pages that no row's window reaches any more are given back
    for s, (m, x) in enumerate(zip(b.new, b.kv)):
        b.pages[s, :max(0, x - m - window + 1) // b.page] = -1
    check(b, window=window)


@pytest.mark.parametrize("dtype", TYPES)
def test_scales(dtype):
    for scale in (1e-6, 0.03, 1.0, 5.0):
        check(Batch4([2, 30], [70, 100], 4, 4, 64, dtype), scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", [[1, 4, 70, 1], [100, 90, 300, 64]])
def test_every_position_has_its_part(dtype, hd, new):
    """Equal scores: the log sum is the log of the number of positions seen, which no lost or doubled one leaves as it is; and one score far
    above the others gives that position's value, bit for bit."""
    kv = [1000, 513, 300, 64]
    b = Batch4(new, kv, 4, 2, hd, dtype)
    b.q.zero_()
    _, lse = check(b)
    at = [x - m + i for m, x in zip(b.new, b.kv) for i in range(m)]
    count = torch.tensor([[float(p + 1)] for p in at])
    assert (torch.exp(lse.cpu()[:b.rows].double()) - count).abs().max() < 0.1
    rng = np.random.default_rng(1)
    b = Batch4(new, kv, 4, 2, hd, dtype)
    b.k_codes.zero_()
    b.k_scales.fill_(127)
    want, row = torch.full((b.rows, 4, hd), math.nan, dtype=dtype), 0
    for s, (m, x) in enumerate(zip(b.new, b.kv)):
        picks = rng.choice(x, size=hd, replace=x < hd)                 # component c of the keys marks position picks[c]
        axis = {}
        for c, p in enumerate(picks):
            axis[int(p)] = c
        for p, c in axis.items():
            b.k_codes[b.slot(s, p)][:, c // 2] |= 7 << 4 * (c % 2)      # 6
        for i in range(m):
            seen = [p for p in axis if p <= x - m + i]
            if seen:
                p = seen[rng.integers(len(seen))]
                b.q[row] = 0
                b.q[row, :, axis[p]] = 64.0                            # a score of 384, the others 0
                want[row] = b.v_cache[b.slot(s, p)].repeat_interleave(2, 0).to(dtype)
            row += 1
    some = ~want.isnan().any(-1)
    assert some.sum() > 150
    d = b.cuda()
    for e, back in variants(d):
        assert torch.equal(back(call(e, scale=1.0)[0]).cpu()[:b.rows][some], want[some])


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_see_nothing(dtype):
    b = Batch4([5, 3, 70, 2], [2, 0, 60, 40], 4, 2, 64, dtype, spare=8)       # kv below the rows: the first ones have no position
    b.pages[3, :] = -1                                                        # a sequence without any page
    check(b)
    check(Batch4([5, 3, 300, 2], [2, 0, 260, 40], 8, 2, 64, dtype))
    check(Batch4([1, 1], [0, 33], 4, 2, 64, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [4, 16])
def test_pages_that_are_not_there(dtype, heads):
    """Holes, numbers that are no page's, lengths behind the table."""
    b = Batch4([3, 70, 1, 2], [200, 170, 300, 90], heads, 2, 128, dtype, spare=4)
    b.pages[0, 3], b.pages[0, 11], b.pages[1, 0], b.pages[1, 5] = -1, b.n_pages, 2 ** 31 - 1, -2 ** 31
    b.pages = b.pages[:, :15].contiguous()
    check(b)
    b.kv_len[2] = 2 ** 31 - 1                                                 # far behind its pages: all of them are seen
    b.kv[2] = 15 * 16 + 1
    b.kv_len[3] = -5
    b.kv[3] = 0
    check(b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bad", [252, 253, 254, 255])
@pytest.mark.parametrize("heads", [4, 8])
def test_what_is_not_seen_has_no_part(dtype, hd, bad, heads):
    """The largest numbers and NaN in free slots, in other sequences' pages, outside the window and in later tokens."""
    def spoil(d, where):
        d.k_scales[where], d.v_scales[where], d.k_codes[where], d.v_codes[where] = bad, bad, 0x7f, 0xf7

    b = Batch4([1, 60, 4, 140], [90, 77, 30, 140], heads, 2, hd, dtype)
    ref = attention64(b)
    d = b.cuda()
    used = torch.zeros(b.n_pages, b.page, dtype=torch.bool)
    for s in range(4):
        for p in range(b.kv[s]):
            used[b.slot(s, p)] = True
    spoil(d, ~used.cuda())
    check(b, d=d, ref=ref)
    # the last tokens of the two runs, and one in the middle: rows before them are as they were
    for s, back in ((1, 1), (1, 40), (3, 1), (3, 100)):
        spoil(d, b.slot(s, b.kv[s] - back))
    first, tol, ltol = b.rows - 140 - 4 - 60, *limits(b, *ref)
    for e, back in variants(d):
        out, lse = map(back, call(e))
        for lo, hi in ((0, first + 60 - 40), (first + 60, first + 64), (first + 64, first + 64 + 40)):
            assert ((out.cpu().double() - ref[0]).abs() <= tol)[lo:hi].all()
            assert ((lse.cpu().double() - ref[1]).abs() <= ltol)[lo:hi].all()
        if bad >= 253:
            assert out[first + 60 - 40:first + 60].isnan().all() and out[first + 64 + 40:].isnan().all() and lse[first + 64 + 40:].isnan().all()
    # outside the window
    b = Batch4([1, 60, 4, 140], [90, 77, 30, 140], heads, 2, hd, dtype)
    ref = attention64(b, window=20)
    d = b.cuda()
    spoil(d, b.slot(3, 50))
    tol, ltol = limits(b, *ref)
    clean = [r for r in range(b.rows) if not (r >= 65 and 50 <= r - 65 < 70)]
    for e, back in variants(d):
        out, lse = map(back, call(e, window=20))
        assert ((out.cpu().double() - ref[0]).abs() <= tol)[clean].all() and ((lse.cpu().double() - ref[1]).abs() <= ltol)[clean].all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,kv", [([1, 40], [90, 60]), ([200, 90], [200, 300]), ([3, 1], [2500, 700])])
def test_values_that_are_nan(dtype, hd, new, kv):
    """They stay in their 32 components, and in the rows that see them; everything else is as exact as it was."""
    b = Batch4(new, kv, 4, 4, hd, dtype)
    ref = attention64(b)
    tol, ltol = limits(b, *ref)
    d = b.cuda()
    hit = torch.zeros_like(ref[0], dtype=torch.bool)
    row = 0
    for s, (m, x) in enumerate(zip(new, kv)):
        for p, h, block in ((17, 0, hd // 32 - 1), (x - 1, 1, 0), (x // 2, 3, 1), (x // 2, 3, 0)):
            d.v_scales[b.slot(s, p)][h, block] = 255
            d.v_codes[b.slot(s, p)][h, 16 * block:16 * block + 16] = 0
            hit[row + max(0, p - (x - m)):row + m, h, 32 * block:32 * block + 32] = True
        row += m
    for e, back in variants(d):
        out, lse = map(back, call(e))
        o = out.cpu().double()
        assert o[hit].isnan().all() and ((o - ref[0]).abs() <= tol)[~hit].all() and ((lse.cpu().double() - ref[1]).abs() <= ltol).all()


@pytest.mark.parametrize("new,kv", [([1, 4, 2], [200, 130, 64]), ([150, 90], [200, 90])])
def test_the_largest_queries(new, kv):
    """Components next to fp32's largest number, above bf16's: their terms are finite."""
    b = Batch4(new, kv, 4, 2, 64, F32)
    b.k_scales[:] = 127 - 125
    b.renew()
    b.q[..., 5] = torch.where(b.q[..., 5] > 0, 3.4028e38, -3.4025e38)
    check(b, scale=float(np.float32(math.log(2.0))))


@pytest.mark.parametrize("dtype", TYPES)
def test_wide_ranges_of_scales(dtype):
    """Blocks of 2^-20 to 2^6 beside each other, as keys and as values."""
    b = Batch4([3, 90, 1], [700, 200, 40], 4, 2, 128, dtype)
    g = torch.Generator().manual_seed(3)
    b.k_scales.copy_(torch.randint(107, 129, b.k_scales.shape, generator=g))
    b.v_scales.copy_(torch.randint(107, 133, b.v_scales.shape, generator=g))
    b.renew()
    check(b)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_and_split(dtype):
    """Few rows over many positions (cut into parts and joined), alone and beside short sequences."""
    check(Batch4([1], [4100], 8, 2, 128, dtype, page=64))
    check(Batch4([4, 1, 1, 2], [3000, 5, 1, 700], 4, 1, 64, dtype, page=32))
    check(Batch4([20, 1], [2500, 2000], 4, 4, 128, dtype, page=16), window=1500)


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_that_differ_a_hundredfold(dtype):
    check(Batch4([1, 1, 2, 1, 1, 1, 1], [60, 6000, 1500, 300, 3000, 100, 40], 32, 32, 64, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_sequences(dtype):
    rng = np.random.default_rng(5)
    new = rng.integers(0, 4, 150)
    check(Batch4(new.tolist(), (new + rng.integers(0, 120, 150)).tolist(), 4, 2, 64, dtype, pad=5))
    check(Batch4([1] * 300, rng.integers(1, 50, 300).tolist(), 2, 2, 64, dtype))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page,window", [(16, 0), (20, 0), (16, 70)])
@pytest.mark.parametrize("heads,kv_heads,new,ctx", [(32, 8, (5, 8), (0, 900)), (16, 16, (17, 32), (0, 300)), (24, 8, (0, 16), (0, 200)), (7, 1, (3, 20), (300, 3000)), (16, 2, (1, 8), (0, 100))])
def test_tiles_of_32_rows(dtype, hd, page, window, heads, kv_heads, new, ctx):
    """Drafts of sequences that share heads, and short runs."""
    rng = np.random.default_rng(heads)
    new = rng.integers(new[0], new[1] + 1, 13)
    check(Batch4(new.tolist(), (new + rng.integers(ctx[0], ctx[1] + 1, 13)).tolist(), heads, kv_heads, hd, dtype, page=page, pad=3), window=window)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("seqs,heads,kv_heads,new,page", [(40, 4, 4, 16, 16), (70, 8, 8, 16, 16), (130, 16, 4, 4, 20), (40, 64, 32, 16, 16), (70, 32, 16, 16, 20), (261, 4, 1, 4, 16), (300, 2, 2, 1, 16), (700, 8, 2, 4, 16)])
def test_tiles_that_are_not_cut(dtype, seqs, heads, kv_heads, new, page):
    """Whole tiles, of sequences of one tile each and a few without any, more than a look finds."""
    rng = np.random.default_rng(seqs)
    n = np.where(rng.random(seqs) < 0.1, 0, new)
    b = Batch4(n.tolist(), (n + rng.integers(0, 150, seqs)).tolist(), heads, kv_heads, 64, dtype, page=page, pad=2)
    check(b)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("seqs", [5, 66, 130])
def test_long_runs_that_are_not_cut(hd, seqs):
    rng = np.random.default_rng(seqs)
    new = np.where(rng.random(seqs) < 0.1, 0, rng.choice([17, 32, 33, 70], seqs))
    group = 8 if seqs < 100 else 4
    b = Batch4(new.tolist(), (new + rng.integers(0, 40, seqs)).tolist(), group, 1, hd, BF16, pad=1)
    d = b.cuda()
    ref = attention64(b)
    e = object.__new__(Batch4)                             # so many heads that every tile is one part, whatever the table's width
    times = 64
    e.__dict__ = dict(d.__dict__, heads=times * group, kv_heads=times, **{n: getattr(d, n).repeat_interleave(times, 2) for n in NAMES})
    e.q = d.q.repeat(1, times, 1)
    wide = long_runs(e) or e
    out, lse = call(wide, out=torch.full_like(e.q, 7.0))
    tol, ltol = limits(b, *ref)
    r = b.rows
    o, z = out.unflatten(1, (times, group)), lse.unflatten(1, (times, group))
    assert torch.equal(o, o[:, :1].expand_as(o)) and torch.equal(z[:r], z[:r, :1].expand_as(z[:r]))
    assert ((o[:r, 0].cpu().double() - ref[0][:r]).abs() <= tol[:r]).all() and ((z[:r, 0].cpu().double() - ref[1][:r]).abs() <= ltol[:r]).all()
    assert (out[r:] == 7.0).all()


@pytest.mark.parametrize("seqs,kv_heads,most", [(65, 2, 900), (130, 2, 600), (530, 1, 400), (4096, 1, 40)])
def test_many_sequences_in_parts(seqs, kv_heads, most):
    rng = np.random.default_rng(seqs)
    new = rng.integers(0, 3, seqs)
    check(Batch4(new.tolist(), (new + rng.integers(0, most, seqs)).tolist(), 3 * kv_heads, kv_heads, 64, BF16, pad=3))


def test_many_long_runs_in_parts():
    rng = np.random.default_rng(1)
    new = np.where(rng.random(70) < 0.2, 0, rng.integers(30, 60, 70))
    check(Batch4(new.tolist(), (new + rng.integers(0, 700, 70)).tolist(), 2, 1, 64, F16, pad=3))
    check(Batch4(new.tolist(), (new + rng.integers(0, 60, 70)).tolist(), 4, 2, 128, BF16, pad=3))           # (one part each)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page,window", [(16, 0), (20, 0), (64, 100)])
@pytest.mark.parametrize("heads,kv_heads", [(8, 8), (14, 2)])
def test_long_runs_in_fp32(hd, page, window, heads, kv_heads):
    check(Batch4([700, 0, 1, 600], [900, 30, 40, 600], heads, kv_heads, hd, F32, page=page, pad=3, seed=hd), window=window)


def test_prompts_beside_tokens():
    check(Batch4([1, 300, 1, 0, 64, 1, 5], [400, 300, 20, 7, 200, 1, 90], 8, 2, 128, BF16, pad=3))
    check(Batch4([1, 300, 1, 0, 64, 1, 5], [400, 300, 20, 7, 200, 1, 90], 8, 8, 64, F16, pad=3), window=50)


def test_strided_rows():
    b = Batch4([3, 20], [50, 60], 4, 2, 128, BF16)
    d = b.cuda()
    ref, _ = call(d)
    whole = torch.zeros((b.n, 9, 128), dtype=BF16, device="cuda")
    whole[:, 2:6] = d.q
    out = torch.full((4, b.n, 128), 3.0, dtype=BF16, device="cuda").transpose(0, 1)
    pool, place = d.pool(), (d.pages, d.q_start, d.kv_len)
    got, _ = binding.ppd_paged_attention_fp4(whole[:, 2:6], *pool, *place, out=out)
    assert got is out and torch.equal(got, ref)
    # in place
    q = d.q.clone()
    assert torch.equal(binding.ppd_paged_attention_fp4(q, *pool, *place, out=q)[0], ref)
    # keys and values in one tensor, as pages of both
    both, scales = torch.stack([d.k_codes, d.v_codes], 1), torch.stack([d.k_scales, d.v_scales], 2)
    got, _ = binding.ppd_paged_attention_fp4(d.q, both[:, 0], scales[:, :, 0], both[:, 1], scales[:, :, 1], *place)
    assert torch.equal(got, ref)
    # a table that is part of a wider one
    wide = torch.full((2, 100), 3, dtype=torch.int32, device="cuda")
    wide[:, :d.pages.shape[1]] = d.pages
    got, _ = binding.ppd_paged_attention_fp4(d.q, *pool, wide[:, :d.pages.shape[1]], d.q_start, d.kv_len)
    assert torch.equal(got, ref)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[1, 1], [70, 90]])
def test_lengths_behind_the_table(dtype, new):
    """A row behind the table's last place sees what the table has, up to the largest length; with a window, what of it is left."""
    b = Batch4(new, [160, 160], 4, 2, 64, dtype, page=16)
    d = b.cuda()
    e = long_runs(d)
    for x in (d, e) if e is not None else (d,):
        x.pages[:, 10:] = -1
        room = x.pages.shape[1] * 16
        want = []
        for length in (room + max(new), 2 ** 31 - 1):
            x.kv_len.fill_(length)
            for window in (0, 2 ** 31 - 1):
                want.append([t.clone() for t in call(x, window=window)])
        assert not want[0][0][:b.rows].isnan().any() and torch.isfinite(want[0][1][:b.rows]).all()
        for w in want[1:3]:
            # (the same positions; a window that long may leave out the first of them, where lengths are largest)
            assert all(torch.equal(x[:b.rows], y[:b.rows]) for x, y in zip(w, want[0]))
        out, lse = call(x, window=5)
        assert (out[:b.rows] == 0).all() and torch.isinf(lse[:b.rows]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_same_bits_every_time(dtype):
    for new in ([1, 3, 40, 1], [1, 3, 300, 1]):
        b = Batch4(new, [2000, 800, 390, 1500], 8, 2, 128, dtype).cuda()
        b = long_runs(b) or b
        out, lse = call(b)
        for _ in range(5):
            o, z = call(b)
            assert torch.equal(o, out) and torch.equal(z, lse)


def test_offsets_beyond_32_bits():
    n_pages = (1 << 32) // (64 * 8 * 64) + 80
    b = Batch4([3, 50], [150, 130], 16, 8, 128, BF16, page=32)
    codes = torch.zeros((n_pages, 64, 8, 64), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n_pages, 64, 8, 4), dtype=torch.uint8, device="cuda")
    for new in ([3, 50], [150, 130]):
        d = b.cuda()
        d.n = sum(new)
        d.new, d.q_start = new, torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
        d.q = torch.randn((sum(new), 16, 128), device="cuda").to(BF16)
        move = torch.arange(n_pages - 2 * b.n_pages, n_pages, 2)[:b.n_pages]
        far = codes[:, :32], scales[:, :32], codes[:, 32:], scales[:, 32:]
        for t, x in zip(far, d.pool()):
            t[move.cuda()] = x
        ref, rl = call(d)
        d.pages = torch.where(d.pages >= 0, move.int().cuda()[d.pages.clamp(min=0).long()], -1)
        d.k_codes, d.k_scales, d.v_codes, d.v_scales = far
        out, lse = call(d)
        assert torch.equal(out, ref) and torch.equal(lse, rl)
        d.pages = torch.cat([d.pages, torch.full((2, 5000), -1, dtype=torch.int32, device="cuda")], 1)      # the kernel for long runs, where these are
        tol, ltol = limits(b, ref.cpu().double(), rl.cpu().double(), torch.full(ref.shape, 5.0), torch.full(rl.shape, 40.0))
        out, lse = call(d)
        assert ((out - ref).cpu().double().abs() <= 2 * tol).all() and ((lse - rl).cpu().double().abs() <= 2 * ltol).all()


def test_streams_replays_and_growing_lengths():
    """Captured once for a table's worth of positions; lengths grow from replay to replay, two graphs live side by side."""
    b = Batch4([2, 1, 1], [40, 700, 3], 8, 2, 128, BF16, extra_pages=4, spare=30).cuda()
    free = [p for p in range(b.n_pages) if p not in b.pages.flatten().tolist()]
    for s in range(3):
        for i in range(b.pages.shape[1]):
            if int(b.pages[s, i]) < 0 and free:
                b.pages[s, i] = free.pop()
    c = Batch4([20, 30], [900, 30], 8, 2, 128, BF16, seed=5).cuda()
    e = Batch4([200, 1, 90], [2900, 5, 700], 8, 2, 128, F16, extra_pages=600).cuda()
    for s in range(3):
        e.pages[s] = torch.randint(0, e.n_pages, (e.pages.shape[1],), dtype=torch.int32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ref, _ = call(b)
    got, _ = call(b, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(ref, got)
    graphs = []
    for x in (b, c, e):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call(x)
        graphs.append((g, x, out))
    for i in range(4):
        for g, x, (out, lse) in graphs:
            x.kv_len += 0 if x is c else 1
            x.q.copy_(torch.randn_like(x.q))
            g.replay()
            o, z = out.clone(), lse.clone()
            torch.cuda.synchronize()
            want, wz = call(x)
            assert torch.equal(o, want) and torch.equal(z, wz)


def test_scratch_memory_of_the_callers():
    """What lies in it does not matter, and no byte behind it is touched."""
    for dtype, new, kv in ((BF16, [1, 2], [3000, 700]), (F16, [200, 90], [2500, 700]), (F32, [4, 1], [900, 2000])):
        b = Batch4(new, kv, 8, 2, 128, dtype).cuda()
        b = long_runs(b) or b
        ref, rl = call(b)
        sizes = binding._paged_args_fp4(*b.pool(), b.pages, b.q_start, b.kv_len, dtype, b.n)[2]
        need = binding._attention_fp4_workspace(sizes, 8)
        assert need > 0
        for fill in (0, 0xff, 0x55):
            w = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda")
            out, lse = call(b, workspace=w[:need])
            assert torch.equal(out, ref) and torch.equal(lse, rl) and (w[need:] == fill).all()
        with pytest.raises(binding.PPDError):
            call(b, workspace=w[:need - 1])


@pytest.mark.parametrize("starts", [[0, 20, 10, 30], [30, 20, 10, 0], [0, 30, -7, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [0, 30] * 30])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kv", [90, 700])
def test_rows_that_are_no_runs(starts, dtype, kv):
    """Where q_start decreases it is undefined what the rows hold; what is written lies in the outputs."""
    b, seqs = Batch4([30], [kv], 16, 2, 64, dtype, spare=5).cuda(), len(starts) - 1
    start, kv_len = torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.full((seqs,), kv, dtype=torch.int32, device="cuda")
    outs = torch.full((40, 16, 64), 5.0, device="cuda").to(dtype)
    for wide in (0, 3000):                                                     # (in a wide table the three sequences are long runs)
        pages = torch.cat([b.pages, torch.full((1, wide), -1, dtype=torch.int32, device="cuda")], 1).repeat(seqs, 1).contiguous()
        binding.ppd_paged_attention_fp4(b.q, *b.pool(), pages, start, kv_len, out=outs[5:-5])
        torch.cuda.synchronize()
        assert (outs[:5] == 5.0).all() and (outs[-5:] == 5.0).all()


@pytest.mark.parametrize("dtype,heads,kv_heads,hd,new", [(BF16, 32, 8, 128, 1), (F32, 8, 4, 64, 2), (F16, 12, 12, 64, 1), (BF16, 80, 16, 128, 3), (F16, 32, 8, 64, 8), (BF16, 64, 8, 128, 6)])
@pytest.mark.parametrize("page,window", [(16, 0), (20, 0), (16, 9000)])
def test_more_than_the_caches_hold(dtype, heads, kv_heads, hd, new, page, window):
    """Lengths of more than 320 MB together, which four heads a workgroup read; each sequence by itself, read by one head a workgroup, gives the same but
    for the order of sums.  (The sequences share pages.)"""
    rng = np.random.default_rng(heads)
    kv = rng.integers(8000, 17000, int(330e6 / (12500 * kv_heads * 2 * 17 * hd / 32)) + 2)
    kv[1], kv[2] = 30, 0
    if window:
        kv = np.concatenate([kv, kv])
    n_pages, seqs = 300, len(kv)
    g = torch.Generator(device="cuda").manual_seed(heads)
    pool = []
    for _ in range(2):
        pool.append(torch.randint(0, 256, (n_pages, page, kv_heads, hd // 2), generator=g, device="cuda", dtype=torch.uint8))
        pool.append(torch.randint(122, 128, (n_pages, page, kv_heads, hd // 32), generator=g, device="cuda", dtype=torch.uint8))
    pool[3][7, 3, 1, 0] = 255                                                  # NaN where many see it
    pages = torch.randint(0, n_pages, (seqs, -(-int(kv.max()) // page)), generator=g, device="cuda", dtype=torch.int32)
    pages[0, 5] = -1
    q = torch.randn((seqs * new, heads, hd), generator=g, device="cuda").to(dtype)
    q_start = (torch.arange(seqs + 1, device="cuda") * new).int()
    kv_len = torch.from_numpy(kv).int().cuda()
    out, lse = binding.ppd_paged_attention_fp4(q, *pool, pages, q_start, kv_len, window=window, want_lse=True)
    for s in range(seqs):
        r = slice(s * new, s * new + new)
        o, z = binding.ppd_paged_attention_fp4(q[r], *pool, pages[s:s + 1], q_start[:2], kv_len[s:s + 1], window=window, want_lse=True)
        torch.cuda.synchronize()
        # both as far off as a score of at most 6 * 3 * hd * 2^0 / sqrt(hd) may be, see limits; values are at most 6
        w = ((QUERY_TERMS[dtype] * hd + 8) * 18 * hd ** 0.5 + WEIGHT_TERMS[dtype] * int(kv[s]) + 16) * 2.0 ** -24
        tol = 2 * (6 * (2 * w + 2.0 ** (-9 * WEIGHT_TERMS[dtype])) + 6 * HALF_STEP[dtype])
        assert torch.equal(o.isnan(), out[r].isnan()) and torch.equal(torch.isinf(z), torch.isinf(lse[r]))
        assert ((o - out[r]).float().abs().nan_to_num() <= tol).all() and ((z - lse[r]).abs().nan_to_num() <= 2 * (w + 40 * 2.0 ** -23)).all()


class Large:
    """Lengths of more than 320 MB together over pages that sequences share, as in test_more_than_the_caches_hold."""

    def __init__(self, dtype, heads, kv_heads, hd, new, page, window):
        rng = np.random.default_rng(hd + heads + new)
        kv = rng.integers(8000, 17000, int(400e6 / (12500 * kv_heads * 2 * 17 * hd / 32)) + 2)
        kv[1], kv[2] = 30, 0
        self.kv = np.concatenate([kv, kv]) if window else kv
        self.dtype, self.heads, self.kv_heads, self.hd, self.new, self.page, self.window, self.n_pages = dtype, heads, kv_heads, hd, new, page, window, 300
        self.pages = torch.from_numpy(rng.integers(0, self.n_pages, (len(self.kv), -(-int(self.kv.max()) // page)))).int()
        self.pages[0, 5], self.pages[-1, 250], self.pages[-1, 251] = -1, self.n_pages, -7
        lo = np.maximum(self.kv - new + 1 - window, 0) if window else 0
        blocks = np.maximum(self.kv - lo, 0) / 64
        assert blocks.sum() * 64 * kv_heads * (hd + hd // 16) > 320e6          # (so that workgroups have four heads)
        # Parts of all tiles (of 16 rows, or of 32) have about the same length, of 2048 / kv_heads parts at most together: positions of one, and parts of one tile.
        self.longest = 64 * (math.ceil(-(-new * heads // kv_heads // 16) * (blocks + 2).sum() / (2048 // kv_heads)) + 1)
        self.parts = 2048 // kv_heads

    def call(self, q, k_codes, k_scales, v_codes, v_scales, scale):
        up = lambda t: t.cuda()  # noqa: E731
        q_start = (torch.arange(len(self.kv) + 1) * self.new).int()
        out, lse = binding.ppd_paged_attention_fp4(up(q), up(k_codes), up(k_scales), up(v_codes), up(v_scales), up(self.pages), up(q_start), up(torch.from_numpy(self.kv).int()),
                                                   scale=scale, window=self.window, want_lse=True)
        torch.cuda.synchronize()
        return out.cpu().double(), lse.cpu().double()

    def weights_off(self, reach):
        """limits' w, but for the sums over positions: those of a part, and then of the parts (three roundings each)."""
        return ((QUERY_TERMS[self.dtype] * self.hd + 8) * reach + WEIGHT_TERMS[self.dtype] * self.longest + 3 * self.parts + 16) * 2.0 ** -24


LARGE = pytest.mark.parametrize("dtype,heads,kv_heads,hd,new", [(BF16, 32, 8, 128, 1), (F32, 8, 4, 64, 2), (F16, 12, 12, 64, 1), (F32, 16, 16, 128, 1), (BF16, 80, 16, 128, 3), (F16, 32, 8, 64, 8),
                                                              (BF16, 64, 8, 128, 6)])
LARGE_PAGES = pytest.mark.parametrize("page,window", [(16, 0), (20, 0), (16, 9000)])


@LARGE
@LARGE_PAGES
@pytest.mark.parametrize("score", [0.0, 87 / 64])
def test_every_position_of_more_than_the_caches_hold(dtype, heads, kv_heads, hd, new, page, window, score):
    """Positions of two kinds, with scores 0 and -score: the log sum tells how many there are of each, and component c of the values, 6 in pages c modulo hd and else 0,
    how many of these.  With equal scores the counts are exact; the other weight, e^-1.359, is no bf16 number by 1/267 of it, nearly the most that there is."""
    x = Large(dtype, heads, kv_heads, hd, new, page, window)
    q = torch.zeros(len(x.kv) * new, heads, hd, dtype=dtype)
    q[..., 33] = score
    k_codes, v_codes = (torch.zeros(x.n_pages, page, kv_heads, hd // 2, dtype=torch.uint8) for _ in "kv")
    scales = torch.full((x.n_pages, page, kv_heads, hd // 32), 127, dtype=torch.uint8)
    k_codes[1::2, ..., 16] = 10 << 4                                           # (component 33: -1)
    for p in range(x.n_pages):
        v_codes[p, ..., p % hd // 2] = 7 << 4 * (p % hd % 2)
    out, lse = x.call(q, k_codes, scales, v_codes, scales, 1.0)
    of_kind = torch.tensor([1.0, math.exp(-score)], dtype=torch.float64)[torch.arange(hd) % 2]
    for s, kv in enumerate(x.kv.tolist()):
        page_of = x.pages[s][torch.arange(max(kv, 1)) // page]
        bucket = torch.where((page_of >= 0) & (page_of < x.n_pages), page_of % hd, hd)
        for i in range(new):
            at, r = kv - new + i, s * new + i
            if at < 0:
                assert (out[r] == 0).all() and (lse[r] == -math.inf).all()
                continue
            count = torch.bincount(bucket[max(0, at - window + 1) if window else 0:at + 1], minlength=hd + 1)[:hd].double()
            total = float((count * of_kind).sum())
            if score == 0:
                # exact sums; the reciprocal, the product, and the rounding to the type
                assert (torch.exp(lse[r]) - total).abs().max() < 0.25
                off = 4 * 2.0 ** -24
            else:
                w = x.weights_off(score)
                assert (lse[r] - math.log(total)).abs().max() <= w + math.log(total) * 2.0 ** -23
                off = 2 * w + 2.0 ** (-9 * WEIGHT_TERMS[dtype])
            want = 6 * count * of_kind / total
            assert ((out[r] - want).abs() <= want * (off + HALF_STEP[dtype] * (1 + 2.0 ** -9))).all(), (s, i, float(((out[r] - want).abs() / want.clamp(min=1e-9)).max()))


@LARGE
@LARGE_PAGES
def test_more_than_the_caches_hold_against_64_bits(dtype, heads, kv_heads, hd, new, page, window):
    """Some sequences and heads of such a batch: holes in the table, a value that is NaN, the first heads and the last."""
    x = Large(dtype, heads, kv_heads, hd, new, page, window)
    g = torch.Generator().manual_seed(heads)
    codes = [torch.randint(0, 256, (x.n_pages, page, kv_heads, hd // 2), generator=g, dtype=torch.uint8) for _ in "kv"]
    scales = [torch.randint(122, 128, (x.n_pages, page, kv_heads, hd // 32), generator=g, dtype=torch.uint8) for _ in "kv"]
    scales[1][7, 3, 1, 0] = 255
    q = torch.randn(len(x.kv) * new, heads, hd, generator=g).to(dtype)
    out, lse = x.call(q, codes[0], scales[0], codes[1], scales[1], hd ** -0.5)
    group = heads // kv_heads
    some = [0, 1, 2, 3, kv_heads - 1] if kv_heads > 4 else list(range(kv_heads))
    k, v = (values64(c[:, :, some], z[:, :, some]) for c, z in zip(codes, scales))
    for s in (0, 1, 2, 3, len(x.kv) - 1):
        r = slice(s * new, s * new + new)
        b = object.__new__(Batch4)
        b.__dict__ = dict(new=[new], kv=[int(x.kv[s])], heads=len(some) * group, kv_heads=len(some), hd=hd, dtype=dtype, page=page, n=new, n_pages=x.n_pages, pages=x.pages[s:s + 1],
                          k_cache=k, v_cache=v, q=q[r].unflatten(1, (kv_heads, group))[:, some].flatten(1, 2))
        ref, z, size, reach = attention64(b, window=window)
        o, l = (t[r].unflatten(1, (kv_heads, group))[:, some].flatten(1, 2) for t in (out, lse))
        assert torch.equal(o.isnan(), ref.isnan()) and torch.equal(torch.isinf(l), torch.isinf(z))
        w = x.weights_off(reach)
        tol = size * (2 * w[..., None] + 2.0 ** (-9 * WEIGHT_TERMS[dtype])) + ref.abs() * HALF_STEP[dtype] * (1 + 2.0 ** -9) + TINY[dtype]
        seen = ~torch.isinf(z)
        assert ((l - z).abs() <= w + z.abs() * 2.0 ** -23)[seen].all(), float((l - z).abs()[seen].max())
        assert ((o - ref).abs() <= tol)[~ref.isnan()].all(), float(((o - ref).abs() / tol)[~ref.isnan()].max())
