"""ppd_paged_append_fp4 against 64 bits: codes and scales have to be the definition's, bit for bit."""
import math

import numpy as np
import pytest
import torch

from fp4_common import NAMES, Batch4, quantised64, values64
from paged_common import HALF_STEP, TINY, append64
from paper_2307_05908_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = float(np.float32(1e-5))                # (what a C float makes of it)


def gains(b, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.2 * torch.randn(b.hd, generator=g)).to(b.dtype) for _ in range(2)]


def call(d, q, q_gain=None, k_gain=None, **kw):
    return binding.ppd_paged_append_fp4(d.k_codes, d.k_scales, d.v_codes, d.v_scales, d.pages, d.q_start, d.kv_len, q, d.k, d.v, q_gain, k_gain, EPS, **kw)


def check(b, norm=(False, False), rotary=0, theta=10000.0, in_place=False, keys_only=False, values=True):
    qg, kg = (g if use else None for g, use in zip(gains(b), norm))
    d = b.cuda()
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    outs = [t if in_place else torch.full_like(t, 7.0) for t in (d.q, d.k, d.v)]
    before = [t.clone() for t in outs]
    got = call(d, None if keys_only else d.q, up(qg), up(kg), rotary_dim=rotary, rope_theta=theta, q_out=None if keys_only else outs[0],
               k_out=outs[1] if values else None, v_out=outs[2] if values else None)
    torch.cuda.synchronize()
    assert (got[0] is None) == keys_only and (got[1] is None) == (got[2] is None) == (not values)
    (q, q_size), (k, _), place = append64(b, qg, kg, EPS, rotary, theta)
    r = b.rows
    if not keys_only:
        # fp32, as ppd_paged_append: 24 roundings of the norm, sine and cosine within 2^-24, two products and a sum; then one to the type
        tol = q_size * 30 * 2.0 ** -24 + q.abs() * HALF_STEP[b.dtype] * (1 + 2.0 ** -10) + TINY[b.dtype]
        bad = (got[0][:r].cpu().double() - q).abs() > tol
        assert not bad.any(), (bad.nonzero()[:5], got[0][:r].cpu().double()[bad][:5], q[bad][:5])
        assert torch.equal(got[0][r:], before[0][r:])
    # every byte of the pages: what was written, and nothing else
    want = {n: getattr(b, n).clone() for n in NAMES}
    (kc, ks), (vc, vs) = quantised64(k), quantised64(b.v[:r])
    for i, (_, slot) in enumerate(place):
        if slot is not None:
            want["k_codes"][slot], want["k_scales"][slot], want["v_codes"][slot], want["v_scales"][slot] = kc[i], ks[i], vc[i], vs[i]
    for n in NAMES:
        bad = getattr(d, n).cpu() != want[n]
        assert not bad.any(), (n, bad.sum(), bad.nonzero()[:5], getattr(d, n).cpu()[bad][:5], want[n][bad][:5])
    if values:
        for x, first, codes, scales in ((got[1], before[1], kc, ks), (got[2], before[2], vc, vs)):
            same = values64(codes, scales).to(b.dtype)
            assert torch.equal(torch.nan_to_num(x[:r].cpu()), torch.nan_to_num(same)) and torch.equal(x[:r].cpu().isnan(), same.isnan())
            assert torch.equal(x[r:], first[r:])
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("norm,share", [((False, False), 1.0), ((True, True), 1.0), ((True, False), 0.5), ((False, True), 0.25)])
def test_types_heads_norms_and_rotated_parts(dtype, hd, norm, share):
    b = Batch4([1, 5, 0, 17], [3, 5, 9, 40], 6, 2, hd, dtype, seed=hd)
    check(b, norm, 0)
    check(b, norm, int(hd * share))
    check(b, norm, 8, values=False)
    check(b, norm, 24)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (8, 1), (5, 5), (40, 8), (33, 11)])
def test_heads(heads, kv_heads):
    check(Batch4([2, 1, 7], [2, 30, 7], heads, kv_heads, 128, BF16, seed=heads), (True, True), 128)
    check(Batch4([2, 1, 7], [2, 30, 7], heads, kv_heads, 64, F32, seed=heads), (True, True), 64)


@pytest.mark.parametrize("page", [1, 3, 16, 20, 256])
def test_pages(page):
    check(Batch4([9, 1, 33], [9, 50, 60], 4, 2, 128, BF16, page=page, seed=page), rotary=128)


@pytest.mark.parametrize("layout,scale_layout", [("phkd", "pkhd"), ("pkhd", "pkhd"), ("hpkd", "phkd"), ("khpd", "hpkd")])
@pytest.mark.parametrize("hd", [64, 128])
def test_orders_of_the_cache(layout, scale_layout, hd):
    check(Batch4([9, 1, 33], [9, 50, 60], 4, 2, hd, F16, layout=layout, scale_layout=scale_layout), (True, True), rotary=hd)


def test_many_rows_and_a_padded_batch():
    check(Batch4([300, 1, 0, 77], [300, 5, 0, 100], 8, 2, 128, BF16, pad=9), rotary=128)
    check(Batch4([700], [900], 2, 2, 64, F32, pad=130), (True, True), rotary=32)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_several_sets_of_rows_a_workgroup(dtype):
    check(Batch4([600, 0, 1], [610, 5, 40], 33, 11, 64, dtype, pad=4), (True, True), rotary=64)
    check(Batch4([500, 300], [500, 300], 21, 7, 128, dtype, page=20), (False, True), rotary=64)
    check(Batch4([1300, 900], [1300, 1000], 3, 1, 64, dtype), (True, False), in_place=True)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("hd,heads,kv_heads", [(128, 2, 1), (128, 1, 1), (128, 4, 2), (128, 8, 4), (128, 14, 1), (64, 2, 1), (64, 12, 4), (64, 16, 8), (64, 5, 5)])
def test_several_tokens_a_workgroup(dtype, hd, heads, kv_heads):
    """Runs that begin and end inside a workgroup's tokens, and padded rows behind the last."""
    check(Batch4([1200, 3, 0, 1, 1, 900, 45], [1210, 3, 4, 1, 70, 1300, 46], heads, kv_heads, hd, dtype, page=20, pad=11), (True, True), rotary=hd)
    b = Batch4([2200, 1], [2200, 30], heads, kv_heads, hd, dtype)
    b.pages[0, 3:60] = -1                                     # no page
    check(b, rotary=hd // 2, keys_only=True)
    check(b, (False, True), rotary=hd // 4, in_place=True)


def test_several_tokens_of_many_sequences():
    rng = np.random.default_rng(1)
    new = rng.choice([0, 1, 3], 4096, p=[0.4, 0.3, 0.3])
    check(Batch4(new.tolist(), (new + rng.integers(0, 20, 4096)).tolist(), 2, 1, 128, BF16, pad=2), rotary=128)


@pytest.mark.parametrize("seqs", [64, 65, 200, 4096])
def test_many_sequences(seqs):
    rng = np.random.default_rng(seqs)
    new = rng.choice([0, 1, 3], seqs, p=[0.6, 0.3, 0.1])
    check(Batch4(new.tolist(), (new + rng.integers(0, 20, seqs)).tolist(), 1, 1, 64, F16, pad=2), rotary=64)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_positions(dtype):
    b = Batch4([3, 5], [10, 12], 4, 2, 128, dtype, page=16)
    b.kv = [1048571, 262147]                                 # the table knows the last page only
    b.kv_len = torch.tensor(b.kv, dtype=torch.int32)
    far = torch.full((2, 1048576 // 16), -1, dtype=torch.int32)
    far[0, (b.kv[0] - 3) // 16], far[1, (b.kv[1] - 5) // 16], far[1, (b.kv[1] - 1) // 16] = b.pages[0, 0], b.pages[1, 0], 4
    b.pages = far
    check(b, (True, True), 128)
    check(b, rotary=128, theta=1e6)


def test_positions_without_a_page():
    b = Batch4([40, 6, 4], [40, 50, 4], 4, 2, 64, BF16, page=16)
    b.pages[0, 1] = -1                       # a hole
    b.pages[1, 2] = b.n_pages                # numbers that are no page's
    b.pages[1, 3] = 2 ** 31 - 1
    b.kv[2] = 2                              # fewer positions than rows: the first two are before the beginning
    b.kv_len = torch.tensor(b.kv, dtype=torch.int32)
    check(b, (True, True), 64)
    b.kv = [100, 1 << 30, 0]                 # behind the table; nothing at all
    b.kv_len = torch.tensor(b.kv, dtype=torch.int32)
    check(b, (True, True), 0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("scale", [0, 9, -9, 100, -100, 108, 109, 110, 111, 112, -108, -109, -110, -111, -112, -113, 123, -122])
def test_borders(dtype, scale):
    """Numbers on the borders between codes and beside them, and largest ones on the borders between scales and beside them."""
    if dtype == F16 and abs(scale) > 9:
        scale //= 11
    b = Batch4([48], [48], 2, 2, 64, dtype, page=20)
    x = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], dtype=torch.float64)
    x = torch.cat([x, -x]) * 2.0 ** scale
    step = 2 * HALF_STEP[dtype]
    for r in range(48):
        for h in range(2):
            off = (1, 1 + step, 1 - step / 2)[r % 3]
            row = torch.cat([x, x.flip(0)]).roll(5 * r + h) * off
            row[(row.abs() == row.abs().max()) & (torch.rand(64) < 0.5)] *= (1, 8 / 7, 0.875)[r // 3 % 3]      # (the largest of 32 may be 7, 8, 6.125)
            b.k[r, h], b.v[r, h] = row.to(dtype), row.flip(0).to(dtype)
    check(b)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_special_values(dtype):
    """Zeros of both signs, the smallest and the largest numbers, and infinities and NaN, which make their 32 numbers NaN and no others."""
    b = Batch4([24], [24], 2, 2, 128, dtype)
    top, least = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    tiny = float(torch.tensor(1, dtype=torch.int32 if dtype == F32 else torch.int16).view(dtype))
    some = [0.0, -0.0, top, -top, least, -least, tiny, -tiny, math.inf, -math.inf, math.nan, top / 2, 2.0 ** -126 if dtype != F16 else tiny, 1.0]
    for t in (b.k, b.v):
        t[0] = 0.0
        t[1] = -0.0
        t[2] = tiny
        t[3] = least * torch.randn(2, 128).clamp(-3, 3)
        t[4] = top
        t[5] = top * torch.rand(2, 128)
        for r in range(6, 20):
            t[r, r % 2, 37 * r % 128] = some[r - 6]
            t[r, 1 - r % 2] *= min(2.0 ** -120, 1.0) if r % 3 else 1.0
    check(b)
    check(b, norm=(False, False), rotary=32)


def test_keys_only_and_strides():
    b = Batch4([9, 1, 33], [9, 50, 60], 8, 2, 128, BF16)
    check(b, (True, True), 128, in_place=True)
    check(b, (True, True), 128, keys_only=True)
    check(Batch4([70, 1], [70, 50], 8, 4, 64, F32), (True, True), 40, in_place=True)
    # one projection's output: queries, keys and values side by side, and a longer row than they fill
    both = torch.randn(b.n, 8 + 2 * 2 + 1, 128).to(BF16)
    ref = Batch4([9, 1, 33], [9, 50, 60], 8, 2, 128, BF16)
    ref.q, ref.k, ref.v = both[:, :8], both[:, 8:10], both[:, 10:12]
    d = ref.cuda()
    whole = both.cuda()
    d.q, d.k, d.v = whole[:, :8], whole[:, 8:10], whole[:, 10:12]
    out = call(d, d.q, rotary_dim=128, want_values=True)
    e = ref.cuda()
    out2 = call(e, e.q, rotary_dim=128, want_values=True)
    assert all(torch.equal(x, y) for x, y in zip(out, out2)) and all(torch.equal(x, y) for x, y in zip(d.pool(), e.pool()))
    assert torch.equal(whole.cpu(), both)
    # heads before tokens
    t = e.q.transpose(0, 1).contiguous().transpose(0, 1)
    out3 = call(e, t, rotary_dim=128, q_out=torch.empty_like(t))[0]
    assert out3.stride() == t.stride() and torch.equal(out3, out2[0])


def test_offsets_beyond_32_bits():
    """Codes more than 2^32 bytes into the cache."""
    n_pages = (1 << 32) // (64 * 8 * 64) + 40
    codes = torch.zeros((n_pages, 64, 8, 64), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n_pages, 64, 8, 4), dtype=torch.uint8, device="cuda")
    kc, vc, ks, vs = codes[:, :32], codes[:, 32:], scales[:, :32], scales[:, 32:]       # keys in the lower half of a page's positions, values in the upper
    pages = torch.tensor([[n_pages - 1, 5, n_pages - 3]], dtype=torch.int32, device="cuda")
    q_start, kv_len = torch.tensor([0, 70], dtype=torch.int32, device="cuda"), torch.tensor([70], dtype=torch.int32, device="cuda")
    k, v = torch.randn((70, 8, 128), device="cuda").to(BF16), torch.randn((70, 8, 128), device="cuda").to(BF16)
    binding.ppd_paged_append_fp4(kc, ks, vc, vs, pages, q_start, kv_len, None, k, v)
    torch.cuda.synchronize()
    for c, s, x in ((kc, ks, k), (vc, vs, v)):
        for got, want in zip((c, s), quantised64(x.cpu())):
            assert torch.equal(torch.cat([got[n_pages - 1], got[5], got[n_pages - 3, :6]]).cpu(), want)
    assert int((scales != 0).any(-1).any(-1).sum()) == 140


def test_streams_and_replays():
    b = Batch4([3, 1], [20, 40], 4, 2, 128, BF16)
    x, y, z = b.cuda(), b.cuda(), b.cuda()
    ref = call(x, x.q, rotary_dim=128, want_values=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = call(y, y.q, rotary_dim=128, want_values=True, stream=side)
    side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(out + y.pool(), ref + x.pool()))
    y = b.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(y, y.q, rotary_dim=128, want_values=True)
    for i in range(3):
        for d in (y, z):
            d.q.copy_(torch.randn(d.q.shape, generator=torch.Generator().manual_seed(i)))
            d.k.copy_(torch.randn(d.k.shape, generator=torch.Generator().manual_seed(9 + i)))
            d.kv_len += 1                                                  # the replays follow the lengths
        graph.replay()
        got, pool = [t.clone() for t in out], [t.clone() for t in y.pool()]
        want = call(z, z.q, rotary_dim=128, want_values=True)
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(got + pool, want + z.pool()))


@pytest.mark.parametrize("starts", [[0, 20, 10, 30], [30, 20, 10, 0], [0, 30, -7, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [0, 30] * 30])
def test_rows_that_are_no_runs(starts):
    """Where q_start decreases it is undefined which rows are written; what is written lies in the outputs and in the pages of the table."""
    b, seqs = Batch4([30], [90], 4, 2, 64, F32, spare=5).cuda(), len(starts) - 1
    start, kv_len = torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.full((seqs,), 90, dtype=torch.int32, device="cuda")
    n = b.n_pages
    pools = [torch.full((n + 4, *t.shape[1:]), 5, dtype=torch.uint8, device="cuda") for t in b.pool()]
    outs = [torch.full((40, t.shape[1], 64), 5.0, device="cuda") for t in (b.q, b.k, b.v)]
    binding.ppd_paged_append_fp4(*(t[2:-2] for t in pools), b.pages.repeat(seqs, 1).contiguous(), start, kv_len, b.q, b.k, b.v, rotary_dim=64, q_out=outs[0][5:-5],
                                 k_out=outs[1][5:-5], v_out=outs[2][5:-5])
    torch.cuda.synchronize()
    mine = torch.zeros(n, dtype=torch.bool)
    mine[b.pages.cpu().flatten().long()] = True
    for t in pools:
        assert (t[:2] == 5).all() and (t[-2:] == 5).all() and (t[2:-2].cpu()[~mine] == 5).all()
    for t in outs:
        assert (t[:5] == 5.0).all() and (t[-5:] == 5.0).all()
