"""ppd_paged_append against 64 bits: heads normalised, rotated and written to their pages."""
import numpy as np
import pytest
import torch

from paged_common import HALF_STEP, TINY, Batch, append64
from paper_2307_05908_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gains(b, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.2 * torch.randn(b.hd, generator=g)).to(b.dtype) for _ in range(2)]


def check(b, norm=(False, False), rotary=0, theta=10000.0, eps=1e-5, in_place=False, keys_only=False):
    qg, kg = (g if use else None for g, use in zip(gains(b), norm))
    d = b.cuda()
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    q_out = d.q if in_place else torch.full_like(d.q, 7.0)
    before_q = q_out.clone()
    k0, v0 = d.k_cache.clone(), d.v_cache.clone()
    got = binding.ppd_paged_append(d.k_cache, d.v_cache, d.pages, d.q_start, d.kv_len, None if keys_only else d.q, d.k, d.v, up(qg), up(kg), eps, rotary, theta,
                                   q_out=None if keys_only else q_out)
    torch.cuda.synchronize()
    assert keys_only == (got is None)
    (q, q_size), (k, k_size), place = append64(b, qg, kg, eps, rotary, theta)

    def near(x, ref, size, turned):
        # fp32: the row's sum of squares (16 products in turn, five levels), root, quotient, two products: 24 roundings; sine and cosine
        # within 2^-22, two products and a sum: 6 more.  Then one rounding to the type.
        tol = size * (24 + (6 if turned else 0)) * 2.0 ** -24 + ref.abs() * HALF_STEP[b.dtype] * (1 + 2.0 ** -10) + TINY[b.dtype]
        bad = (x.cpu().double() - ref).abs() > tol
        assert not bad.any(), (bad.nonzero()[:5], x.cpu().double()[bad][:5], ref[bad][:5])

    if not keys_only:
        near(got[:b.rows], q, q_size, rotary > 0)
        assert torch.equal(got[b.rows:], before_q[b.rows:])
    # every slot of the caches: what was written, and nothing else
    k0, v0, kc, vc = k0.cpu(), v0.cpu(), d.k_cache.cpu(), d.v_cache.cpu()
    written = torch.zeros(b.n_pages, b.page, dtype=torch.bool)
    for r, (_, slot) in enumerate(place):
        if slot is None:
            continue
        written[slot] = True
        near(kc[slot], k[r], k_size[r], rotary > 0)
        assert torch.equal(vc[slot], b.v[r])
    assert torch.equal(kc[~written], k0[~written]) and torch.equal(vc[~written], v0[~written])
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("norm,share", [((False, False), 1.0), ((True, True), 1.0), ((True, False), 0.5), ((False, True), 0.25)])
def test_types_heads_norms_and_rotated_parts(dtype, hd, norm, share):
    b = Batch([1, 5, 0, 17], [3, 5, 9, 40], 6, 2, hd, dtype, seed=hd)
    check(b, norm, 0)
    check(b, norm, int(hd * share))
    check(b, norm, 8)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (8, 1), (5, 5), (40, 8), (33, 11)])
def test_heads(heads, kv_heads):
    check(Batch([2, 1, 7], [2, 30, 7], heads, kv_heads, 128, BF16, seed=heads), (True, True), 128)
    check(Batch([2, 1, 7], [2, 30, 7], heads, kv_heads, 64, F32, seed=heads), (True, True), 64)


@pytest.mark.parametrize("page", [1, 3, 16, 20, 256])
def test_pages(page):
    check(Batch([9, 1, 33], [9, 50, 60], 4, 2, 128, BF16, page=page, seed=page), rotary=128)


@pytest.mark.parametrize("layout", ["phkd", "pkhd", "hpkd", "khpd"])
def test_orders_of_the_cache(layout):
    check(Batch([9, 1, 33], [9, 50, 60], 4, 2, 128, F16, layout=layout), (True, True), rotary=128)


def test_many_rows_and_a_padded_batch():
    check(Batch([300, 1, 0, 77], [300, 5, 0, 100], 8, 2, 128, BF16, pad=9), rotary=128)
    check(Batch([700], [900], 2, 2, 64, F32, pad=130), (True, True), rotary=32)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_several_sets_of_rows_a_workgroup(dtype):
    check(Batch([600, 0, 1], [610, 5, 40], 33, 11, 64, dtype, pad=4), (True, True), rotary=64)
    check(Batch([500, 300], [500, 300], 21, 7, 128, dtype, page=20), (False, True), rotary=64)
    check(Batch([1300, 900], [1300, 1000], 3, 1, 64, dtype), (True, False), in_place=True)


def test_many_sequences():
    rng = np.random.default_rng(3)
    new = rng.integers(0, 3, 200)
    check(Batch(new.tolist(), (new + rng.integers(0, 30, 200)).tolist(), 2, 1, 64, BF16), rotary=64)


@pytest.mark.parametrize("seqs", [64, 65, 128, 1000, 4095, 4096])
def test_as_many_sequences_as_there_may_be(seqs):
    rng = np.random.default_rng(seqs)
    new = rng.choice([0, 1, 3], seqs, p=[0.6, 0.3, 0.1])
    check(Batch(new.tolist(), (new + rng.integers(0, 20, seqs)).tolist(), 1, 1, 64, F16, pad=2), rotary=64)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_positions(dtype):
    """Angles of a million radians, to the last digits of fp32."""
    b = Batch([3, 5], [10, 12], 4, 2, 128, dtype, page=16)
    b.kv = [1048571, 262147]                                 # the table knows the last page only
    b.kv_len = torch.tensor(b.kv, dtype=torch.int32)
    far = torch.full((2, 1048576 // 16), -1, dtype=torch.int32)
    far[0, (b.kv[0] - 3) // 16], far[1, (b.kv[1] - 5) // 16], far[1, (b.kv[1] - 1) // 16] = b.pages[0, 0], b.pages[1, 0], 4
    b.pages = far
    check(b, (True, True), 128)
    check(b, rotary=128, theta=1e6)


def test_positions_without_a_page():
    b = Batch([40, 6, 4], [40, 50, 4], 4, 2, 64, BF16, page=16)
    b.pages[0, 1] = -1                       # a hole
    b.pages[1, 2] = b.n_pages                # numbers that are no page's
    b.pages[1, 3] = 2 ** 31 - 1
    b.kv[2] = 2                              # fewer positions than rows: the first two are before the beginning
    b.kv_len = torch.tensor(b.kv, dtype=torch.int32)
    check(b, (True, True), 64)
    b.kv = [100, 1 << 30, 0]                 # behind the table; nothing at all
    b.kv_len = torch.tensor(b.kv, dtype=torch.int32)
    check(b, (True, True), 0)


def test_in_place_keys_only_and_strides():
    b = Batch([9, 1, 33], [9, 50, 60], 8, 2, 128, BF16)
    check(b, (True, True), 128, in_place=True)
    check(b, (True, True), 128, keys_only=True)
    # one projection's output: queries, keys and values side by side, and a longer row than they fill
    both = torch.randn(b.n, 8 + 2 * 2 + 1, 128).to(BF16)
    ref = Batch([9, 1, 33], [9, 50, 60], 8, 2, 128, BF16)
    ref.q, ref.k, ref.v = both[:, :8], both[:, 8:10], both[:, 10:12]
    d = ref.cuda()
    whole = both.cuda()
    d.q, d.k, d.v = whole[:, :8], whole[:, 8:10], whole[:, 10:12]
    out = binding.ppd_paged_append(d.k_cache, d.v_cache, d.pages, d.q_start, d.kv_len, d.q, d.k, d.v, rotary_dim=128)
    e = ref.cuda()
    out2 = binding.ppd_paged_append(e.k_cache, e.v_cache, e.pages, e.q_start, e.kv_len, e.q, e.k, e.v, rotary_dim=128)
    assert torch.equal(out, out2) and torch.equal(d.k_cache, e.k_cache) and torch.equal(d.v_cache, e.v_cache)
    assert torch.equal(whole.cpu(), both)
    # heads before tokens
    t = e.q.transpose(0, 1).contiguous().transpose(0, 1)
    out3 = binding.ppd_paged_append(e.k_cache, e.v_cache, e.pages, e.q_start, e.kv_len, t, e.k, e.v, rotary_dim=128, q_out=torch.empty_like(t))
    assert out3.stride() == t.stride() and torch.equal(out3, out2)


def test_special_values_are_copied():
    b = Batch([4], [4], 2, 2, 64, BF16)
    b.v[0, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0])
    b.k[1, 1, 5] = float("inf")
    b.q[2, 0, 9] = float("nan")
    d = b.cuda()
    q = binding.ppd_paged_append(d.k_cache, d.v_cache, d.pages, d.q_start, d.kv_len, d.q, d.k, d.v, rotary_dim=0)
    torch.cuda.synchronize()
    bits = lambda t: t.cpu().contiguous().view(torch.int16)  # noqa: E731
    page = int(b.pages[0, 0])
    assert torch.equal(bits(q), bits(b.q)) and torch.equal(bits(d.k_cache[page, :4]), bits(b.k)) and torch.equal(bits(d.v_cache[page, :4]), bits(b.v))


def test_offsets_beyond_32_bits():
    """Pages more than 2^31 elements, and 2^32 bytes, into the cache."""
    n_pages = (1 << 31) // (64 * 8 * 128) + 40
    kc = torch.zeros((n_pages, 64, 8, 128), dtype=BF16, device="cuda")
    vc = kc.view(-1)[:].view(n_pages, 64, 8, 128)                           # keys in the lower half of a page's positions, values in the upper
    k_half, v_half = kc[:, :32], vc[:, 32:]
    pages = torch.tensor([[n_pages - 1, 5, n_pages - 3]], dtype=torch.int32, device="cuda")
    q_start, kv_len = torch.tensor([0, 70], dtype=torch.int32, device="cuda"), torch.tensor([70], dtype=torch.int32, device="cuda")
    k, v = torch.randn((70, 8, 128), device="cuda").to(BF16), torch.randn((70, 8, 128), device="cuda").to(BF16)
    binding.ppd_paged_append(k_half, v_half, pages, q_start, kv_len, None, k, v)
    torch.cuda.synchronize()
    for c, x in ((k_half, k), (v_half, v)):
        assert torch.equal(c[n_pages - 1], x[:32]) and torch.equal(c[5], x[32:64]) and torch.equal(c[n_pages - 3, :6], x[64:])
    assert int((kc != 0).any(-1).any(-1).sum()) == 140


def test_streams_and_replays():
    b = Batch([3, 1], [20, 40], 4, 2, 128, BF16).cuda()
    ref_k, ref_v = b.k_cache.clone(), b.v_cache.clone()
    args = (b.pages, b.q_start, b.kv_len)
    ref = binding.ppd_paged_append(ref_k, ref_v, *args, b.q, b.k, b.v, rotary_dim=128)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k2, v2 = b.k_cache.clone(), b.v_cache.clone()
    side.wait_stream(torch.cuda.current_stream())
    out = binding.ppd_paged_append(k2, v2, *args, b.q, b.k, b.v, rotary_dim=128, stream=side)
    side.synchronize()
    assert torch.equal(out, ref) and torch.equal(k2, ref_k) and torch.equal(v2, ref_v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.ppd_paged_append(b.k_cache, b.v_cache, *args, b.q, b.k, b.v, rotary_dim=128)
    ref_k, ref_v = b.k_cache.clone(), b.v_cache.clone()                    # (a capture writes nothing)
    for i in range(3):
        b.q.copy_(torch.randn_like(b.q)); b.kv_len += 1                    # the replays follow the lengths
        graph.replay()
        got, gk = out.clone(), b.k_cache.clone()
        want = binding.ppd_paged_append(ref_k, ref_v, *args, b.q, b.k, b.v, rotary_dim=128)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(gk, ref_k)


@pytest.mark.parametrize("starts", [[0, 20, 10, 30], [30, 20, 10, 0], [0, 30, -7, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [0, 30] * 30])
def test_rows_that_are_no_runs(starts):
    """Where q_start decreases it is undefined which rows are written; what is written lies in the outputs and in the pages of the table."""
    b, seqs = Batch([30], [90], 4, 2, 64, torch.float32, spare=5).cuda(), len(starts) - 1
    start, kv_len = torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.full((seqs,), 90, dtype=torch.int32, device="cuda")
    n = b.k_cache.shape[0]
    ks, vs = (torch.full((n + 4, *b.k_cache.shape[1:]), 5.0, device="cuda") for _ in range(2))
    outs = torch.full((40, 4, 64), 5.0, device="cuda")
    binding.ppd_paged_append(ks[2:-2], vs[2:-2], b.pages.repeat(seqs, 1).contiguous(), start, kv_len, b.q, b.k, b.v, rotary_dim=64, q_out=outs[5:-5])
    torch.cuda.synchronize()
    mine = torch.zeros(n, dtype=torch.bool)
    mine[b.pages.cpu().flatten().long()] = True
    for t in (ks, vs):
        assert (t[:2] == 5.0).all() and (t[-2:] == 5.0).all() and (t[2:-2].cpu()[~mine] == 5.0).all()
    assert (outs[:5] == 5.0).all() and (outs[-5:] == 5.0).all()
