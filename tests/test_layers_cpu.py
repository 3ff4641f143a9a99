"""What the operators of include/ppd_layers.h refuse, on the CPU: nothing is queued, nothing dereferenced."""
import ctypes

import pytest
import torch

from paper_2307_05908_amd import binding

P = ctypes.c_void_p(4096)
EINVAL, ELIMIT = -1, -6


def cache(**kw):
    a = dict(k=4096, v=4096, k_page=16 * 8 * 64, k_pos=8 * 64, k_head=64, v_page=16 * 8 * 64, v_pos=8 * 64, v_head=64, n_pages=10, page_size=16, n_kv_heads=8,
             head_dim=64, dtype=1)
    a.update(kw)
    return binding.PagedCache(**a)


def batch(**kw):
    a = dict(q_start=4096, kv_len=4096, pages=4096, pages_stride=4, max_pages=4, n_seqs=3, n_tokens=7)
    a.update(kw)
    return binding.PagedBatch(**a)


def rows(**kw):
    a = dict(p=4096, token=16 * 64, head=64)
    a.update(kw)
    return binding.Rows(**a)


BAD_CACHE = [dict(k=None), dict(v=None), dict(k=4100), dict(v=4104), dict(k_page=-64), dict(k_pos=4), dict(v_head=7), dict(v_page=12), dict(n_pages=0),
             dict(page_size=0), dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=0), dict(dtype=3), dict(dtype=-1)]
BAD_BATCH = [dict(q_start=None), dict(kv_len=None), dict(pages=None), dict(pages=4097), dict(n_seqs=0), dict(n_tokens=-1), dict(max_pages=0), dict(pages_stride=3)]
TOO_LARGE = [dict(n_seqs=4097), dict(n_tokens=(1 << 22) + 1), dict(max_pages=(1 << 26) + 1, pages_stride=1 << 27)]
BAD_ROWS = [dict(p=None), dict(p=4104), dict(token=-64), dict(token=12), dict(head=4)]


def attention(c=None, b=None, heads=16, q=None, out=None, lse=None, scale=0.125, window=0, ws=P, size=1 << 40):
    return binding.load_library().ppd_paged_attention(c or cache(), b or batch(), heads, q or rows(), out or rows(), lse, scale, window, ws, size, None)


def append(c=None, b=None, heads=16, q=None, q_out=None, k=None, v=None, qg=None, kg=None, eps=1e-5, rotary=64, theta=1e4):
    return binding.load_library().ppd_paged_append(c or cache(), b or batch(), heads, q or rows(), q_out or rows(p=1 << 20), k or rows(token=512), v or rows(token=512),
                                                   qg, kg, eps, rotary, theta, None)


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_bad_cache(kw):
    assert attention(c=cache(**kw)) == EINVAL and append(c=cache(**kw)) == EINVAL
    n = ctypes.c_uint64(7)
    assert binding.load_library().ppd_paged_attention_workspace(cache(**kw), batch(), 16, ctypes.byref(n)) == EINVAL and n.value == 7


@pytest.mark.parametrize("kw", BAD_BATCH)
def test_bad_batch(kw):
    assert attention(b=batch(**kw)) == EINVAL and append(b=batch(**kw)) == EINVAL


@pytest.mark.parametrize("kw", TOO_LARGE)
def test_too_large(kw):
    assert attention(b=batch(**kw)) == ELIMIT and append(b=batch(**kw)) == ELIMIT


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_bad_rows(kw):
    bad = rows(**kw)
    assert attention(q=bad) == EINVAL and attention(out=bad) == EINVAL
    for name in ("q", "q_out", "k", "v"):
        assert append(**{name: bad}) == EINVAL


def test_bad_attention_arguments():
    assert attention(heads=0) == EINVAL and attention(heads=12) == EINVAL and attention(heads=1032, c=cache(n_kv_heads=8)) == ELIMIT
    assert attention(scale=0.0) == EINVAL and attention(scale=-1.0) == EINVAL and attention(scale=float("nan")) == EINVAL and attention(scale=float("inf")) == EINVAL
    assert attention(scale=3e38) == EINVAL                                                            # (its product with log2 e is not finite)
    assert attention(window=-1) == EINVAL and attention(lse=ctypes.c_void_p(4098)) == EINVAL
    assert attention(out=rows(token=0)) == EINVAL and attention(out=rows(head=0)) == EINVAL          # rows written onto each other


def test_workspace_of_attention_is_checked():
    lib = binding.load_library()
    need = ctypes.c_uint64()
    for heads in (8, 16):
        b = batch(max_pages=1000, pages_stride=1000)
        assert lib.ppd_paged_attention_workspace(cache(), b, heads, ctypes.byref(need)) == 0
        if need.value:
            assert attention(b=b, heads=heads, ws=None) == EINVAL and attention(b=b, heads=heads, size=need.value - 1) == EINVAL
            assert attention(b=b, heads=heads, ws=ctypes.c_void_p(4104)) == EINVAL
    assert lib.ppd_paged_attention_workspace(cache(), batch(), 16, None) == EINVAL


@pytest.mark.parametrize("dtype,tokens,heads", [(0, 1 << 22, 64), (0, 1 << 19, 512), (1, 1 << 22, 512)])
def test_more_workgroups_than_a_launch_may_have(dtype, tokens, heads):
    """Refused, and by the size of its scratch memory already; half of it is not."""
    lib, need = binding.load_library(), ctypes.c_uint64()
    c, q = cache(dtype=dtype, n_kv_heads=heads // 2, k_head=64, v_head=64), rows(token=heads * 64)
    for n, rc in ((tokens, ELIMIT), (tokens // 2, 0)):
        assert lib.ppd_paged_attention_workspace(c, batch(n_tokens=n), heads, ctypes.byref(need)) == rc
    assert attention(c=c, b=batch(n_tokens=tokens), heads=heads, q=q, out=q) == ELIMIT


def test_bad_append_arguments():
    assert append(heads=-1) == EINVAL and append(heads=1025) == ELIMIT
    for r in (-8, 4, 60, 72):
        assert append(rotary=r) == EINVAL
    for theta in (0.0, -2.0, float("nan"), float("inf")):
        assert append(theta=theta) == EINVAL
    for eps in (-1e-5, float("nan"), float("inf")):
        assert append(qg=P, eps=eps) == EINVAL and append(kg=P, eps=eps) == EINVAL
    assert append(qg=ctypes.c_void_p(4100)) == EINVAL and append(kg=ctypes.c_void_p(4100)) == EINVAL
    assert append(c=cache(dtype=0), qg=ctypes.c_void_p(4104)) == EINVAL
    assert append(q=rows(), q_out=rows(head=128)) == EINVAL                                          # in place with other strides
    assert append(q_out=rows(p=1 << 20, token=0)) == EINVAL


@pytest.mark.parametrize("name", ["k_page", "k_pos", "k_head", "v_page", "v_pos", "v_head"])
def test_append_to_pages_that_lie_on_each_other(name):
    assert append(c=cache(**{name: 0})) == EINVAL
    assert append(c=cache(n_pages=1, page_size=1, n_kv_heads=1, **{name: 0}), b=batch(n_tokens=0)) == 0      # (nothing to lie on)


def test_nothing_to_do_is_no_error():
    assert attention(b=batch(n_tokens=0)) == 0 and append(b=batch(n_tokens=0)) == 0


def verify(seqs=3, n=9, vocab=1000, dtype=0, start=P, ids=P, z=P, zs=1000, d=None, ds=0, t=None, u=P, tok=P, acc=P, ws=P, size=1 << 40):
    return binding.load_library().ppd_verify_drafts(seqs, n, vocab, dtype, start, ids, z, zs, d, ds, t, u, tok, acc, ws, size, None)


def test_bad_verify_arguments():
    assert verify(seqs=0) == EINVAL and verify(n=-1) == EINVAL and verify(vocab=0) == EINVAL and verify(dtype=3) == EINVAL and verify(dtype=-1) == EINVAL
    assert verify(seqs=4097) == ELIMIT and verify(n=(1 << 22) + 1) == ELIMIT and verify(vocab=(1 << 24) + 1, zs=1 << 25) == ELIMIT
    for name in ("start", "ids", "z", "u", "tok", "acc"):
        assert verify(**{name: None}) == EINVAL
        assert verify(**{name: ctypes.c_void_p(4098)}) == EINVAL
    assert verify(dtype=1, z=ctypes.c_void_p(4097)) == EINVAL and verify(d=ctypes.c_void_p(4098), ds=1000) == EINVAL
    assert verify(t=ctypes.c_void_p(4097)) == EINVAL
    assert verify(zs=999) == EINVAL and verify(d=P, ds=999) == EINVAL
    n = ctypes.c_uint64()
    lib = binding.load_library()
    assert lib.ppd_verify_drafts_workspace(3, 9, 1000, 0, None) == EINVAL and lib.ppd_verify_drafts_workspace(3, 9, 0, 0, ctypes.byref(n)) == EINVAL
    assert lib.ppd_verify_drafts_workspace(3, 9, 1000, 0, ctypes.byref(n)) == 0
    if n.value:
        assert verify(ws=None) == EINVAL and verify(size=n.value - 1) == EINVAL and verify(ws=ctypes.c_void_p(4104)) == EINVAL


def test_binding_refuses_what_the_library_cannot_see():
    t = torch.zeros
    with pytest.raises(ValueError):           # not on a GPU
        binding.ppd_paged_attention(t(2, 4, 64), t(3, 16, 4, 64), t(3, 16, 4, 64), t(1, 3, dtype=torch.int32), t(2, dtype=torch.int32), t(1, dtype=torch.int32))
    k = t(3, 16, 4, 64)
    i32 = torch.int32
    good = (t(1, 3, dtype=i32), t(2, dtype=i32), t(1, dtype=i32))
    binding._paged_args(k, k, *good, 2)
    for bad in ((k, k.half(), *good), (k, t(3, 16, 4, 32), *good), (k[0], k[0], *good), (k.transpose(2, 3), k.transpose(2, 3), *good),
                (k, k, t(1, 3, dtype=torch.int64), *good[1:]), (k, k, t(2, 3, dtype=i32), *good[1:]), (k, k, good[0], t(3, dtype=i32), good[2]),
                (k, k, t(1, 6, dtype=i32)[:, ::2], *good[1:])):
        with pytest.raises(ValueError):
            binding._paged_args(*bad, 2)
    for q in (t(2, 4, 32), t(3, 4, 64), t(2, 4, 64).half(), t(2, 64, 4).transpose(1, 2), t(2, 64)):
        with pytest.raises(ValueError):
            binding._rows(q, k.dtype, 64, "q", 2)


def test_binding_refuses_scratch_memory_that_is_not_in_a_row():
    """An expanded tensor's bytes are those of its shape, not of its memory."""
    w = torch.zeros(64, dtype=torch.uint8)
    assert binding._scratch(w) == (w.data_ptr(), 64) and binding._scratch(None) == (None, 0) and binding._scratch(w[16:32]) == (w.data_ptr() + 16, 16)
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), w[::2], torch.zeros(8, 8, dtype=torch.uint8).t()[:, :4]):
        with pytest.raises(ValueError):
            binding._scratch(bad)
