"""What the operators around a step refuse, on the CPU: nothing is queued, nothing dereferenced."""
import ctypes
import os
import re

import pytest
import torch

from paper_2307_05908_amd import binding
from test_layers_cpu import BAD_BATCH, BAD_ROWS, EINVAL, ELIMIT, P, TOO_LARGE, batch, rows


def cache(**kw):
    a = dict(k=4096, v=4096, k_scales=4096, v_scales=4096, k_page=16 * 8 * 32, k_pos=8 * 32, k_head=32, v_page=16 * 8 * 32, v_pos=8 * 32, v_head=32,
             ks_page=16 * 8 * 2, ks_pos=16, ks_head=2, vs_page=16 * 8 * 2, vs_pos=16, vs_head=2, n_pages=10, page_size=16, n_kv_heads=8, head_dim=64, dtype=1)
    a.update(kw)
    return binding.PagedCacheFp4(**a)


BAD_CACHE = [dict(k=None), dict(v=None), dict(k_scales=None), dict(v_scales=None), dict(k=4104), dict(v=4097), dict(k_scales=4097), dict(v_scales=4099), dict(k_page=-64),
             dict(k_pos=8), dict(v_head=24), dict(v_page=12), dict(ks_page=3), dict(ks_pos=-2), dict(vs_head=1), dict(vs_pos=5), dict(n_pages=0), dict(page_size=0),
             dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=0), dict(dtype=3), dict(dtype=-1), dict(head_dim=128, k_scales=4098), dict(head_dim=128, ks_head=2)]


def attention(c=None, b=None, heads=16, q=None, out=None, lse=None, scale=0.125, window=0, ws=P, size=1 << 40):
    return binding.load_library().ppd_paged_attention_fp4(c or cache(), b or batch(), heads, q or rows(), out or rows(), lse, scale, window, ws, size, None)


def append(c=None, b=None, heads=16, q=None, q_out=None, k=None, v=None, k_out=None, v_out=None, qg=None, kg=None, eps=1e-5, rotary=64, theta=1e4):
    return binding.load_library().ppd_paged_append_fp4(c or cache(), b or batch(), heads, q or rows(), q_out or rows(p=1 << 20), k or rows(token=512), v or rows(token=512),
                                                       k_out, v_out, qg, kg, eps, rotary, theta, None)


def test_declared_names_are_exported():
    """All of them, with digits in their names or without."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ppd_layers.h")).read()
    names = set(re.findall(r"\b(ppd_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert {n for n in names if re.search(r"\d", n)} == set(binding.FP4_EXPORTS) and names <= {*binding.EXPORTS, *binding.FP4_EXPORTS}
    for n in names:
        assert getattr(binding.load_library(), n) is not None


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_bad_cache(kw):
    assert attention(c=cache(**kw)) == EINVAL and append(c=cache(**kw)) == EINVAL
    n = ctypes.c_uint64(7)
    assert binding.load_library().ppd_paged_attention_fp4_workspace(cache(**kw), batch(), 16, ctypes.byref(n)) == EINVAL and n.value == 7


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
    for name in ("q", "q_out", "k", "v", "k_out", "v_out"):
        assert append(**{name: bad}) == EINVAL


def test_bad_attention_arguments():
    assert attention(heads=0) == EINVAL and attention(heads=12) == EINVAL and attention(heads=1032) == ELIMIT
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert attention(scale=scale) == EINVAL
    assert attention(window=-1) == EINVAL and attention(lse=ctypes.c_void_p(4098)) == EINVAL
    assert attention(out=rows(token=0)) == EINVAL and attention(out=rows(head=0)) == EINVAL          # rows written onto each other
    lib, need = binding.load_library(), ctypes.c_uint64()
    b = batch(max_pages=1000, pages_stride=1000)
    assert lib.ppd_paged_attention_fp4_workspace(cache(), b, 16, ctypes.byref(need)) == 0 and need.value > 0
    assert attention(b=b, ws=None) == EINVAL and attention(b=b, size=need.value - 1) == EINVAL and attention(b=b, ws=ctypes.c_void_p(4104)) == EINVAL
    assert lib.ppd_paged_attention_fp4_workspace(cache(), b, 16, None) == EINVAL


@pytest.mark.parametrize("dtype,tokens,heads", [(0, 1 << 22, 64), (0, 1 << 19, 512), (1, 1 << 22, 512)])
def test_more_workgroups_than_a_launch_may_have(dtype, tokens, heads):
    lib, need = binding.load_library(), ctypes.c_uint64()
    c, q = cache(dtype=dtype, n_kv_heads=heads // 2), rows(token=heads * 64)
    for n, rc in ((tokens, ELIMIT), (tokens // 2, 0)):
        assert lib.ppd_paged_attention_fp4_workspace(c, batch(n_tokens=n), heads, ctypes.byref(need)) == rc
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
    for name, where in (("q_out", "q"), ("k_out", "k"), ("v_out", "v")):
        assert append(**{name: rows(head=128)}) == EINVAL                                            # in place with other strides
        assert append(**{name: rows(p=1 << 20, token=0)}) == EINVAL


@pytest.mark.parametrize("name", [x + y for x in ("k", "v", "ks", "vs") for y in ("_page", "_pos", "_head")])
def test_append_to_pages_that_lie_on_each_other(name):
    assert append(c=cache(**{name: 0})) == EINVAL
    assert append(c=cache(n_pages=1, page_size=1, n_kv_heads=1, **{name: 0}), b=batch(n_tokens=0)) == 0      # (nothing to lie on)


def test_nothing_to_do_is_no_error():
    assert attention(b=batch(n_tokens=0)) == 0 and append(b=batch(n_tokens=0)) == 0 and adjust(n=0) == 0


def plan(counters=P, counters_out=P, held=P, kept=P, wanted=P, n=9, start=P, kv=P, granted=P, seq=P, pos=P, slots=P, **kw):
    a = dict(pages=4096, pages_stride=8, free_pages=4096, max_pages=8, n_pages=100, page_size=16, n_seqs=3)
    a.update(kw)
    return binding.load_library().ppd_paged_plan(binding.PageTable(**a), counters, counters_out, held, kept, wanted, n, start, kv, granted, seq, pos, slots, None)


def test_bad_plan_arguments():
    lib = binding.load_library()
    assert lib.ppd_paged_plan(None, P, P, P, P, P, 9, P, P, P, P, P, P, None) == EINVAL
    for name in ("counters", "counters_out", "held", "wanted", "start", "kv", "granted"):
        assert plan(**{name: None}) == EINVAL
    for name in ("held", "kept", "wanted", "start", "kv", "granted", "seq", "pos"):
        assert plan(**{name: ctypes.c_void_p(4098)}) == EINVAL
    for name in ("counters", "counters_out", "slots"):
        assert plan(**{name: ctypes.c_void_p(4100)}) == EINVAL
    for kw in (dict(pages=None), dict(free_pages=None), dict(pages=4097), dict(free_pages=4098), dict(n_seqs=0), dict(max_pages=0), dict(n_pages=0), dict(page_size=0),
               dict(n=-1), dict(pages_stride=7)):
        assert plan(**kw) == EINVAL
    for kw in (dict(n_seqs=4097), dict(n=(1 << 22) + 1), dict(max_pages=(1 << 26) + 1, pages_stride=1 << 27), dict(max_pages=1 << 19, pages_stride=1 << 19, n_seqs=4096)):
        assert plan(**kw) == ELIMIT


def adjust(seqs=3, n=9, vocab=1000, dtype=0, start=P, ids=P, z=P, zs=1000, out=P, outs=1000, rules=True, **kw):
    a = dict(history=4096, history_stride=50, history_len=4096, prompt_len=4096, repetition=4096, presence=4096, frequency=4096, bias_start=4096, bias_ids=4096, bias=4096,
             mask=4096, mask_stride=32, mask_row=4096, n_bias=5, n_masks=2)
    a.update(kw)
    return binding.load_library().ppd_adjust_logits(seqs, n, vocab, dtype, start, ids, z, zs, out, outs, binding.LogitRules(**a) if rules else None, None)


def test_bad_adjust_arguments():
    assert adjust(rules=False) == EINVAL
    assert adjust(seqs=0) == EINVAL and adjust(n=-1) == EINVAL and adjust(vocab=0) == EINVAL and adjust(dtype=3) == EINVAL and adjust(dtype=-1) == EINVAL
    assert adjust(seqs=4097) == ELIMIT and adjust(n=(1 << 22) + 1) == ELIMIT and adjust(vocab=(1 << 24) + 1, zs=1 << 25, outs=1 << 25, mask_stride=1 << 20) == ELIMIT
    for name in ("start", "z", "out"):
        assert adjust(**{name: None}) == EINVAL and adjust(**{name: ctypes.c_void_p(4098)}) == EINVAL
    assert adjust(ids=ctypes.c_void_p(4097)) == EINVAL and adjust(dtype=1, z=ctypes.c_void_p(4097)) == EINVAL
    assert adjust(zs=999) == EINVAL and adjust(outs=999) == EINVAL and adjust(zs=1008) == EINVAL        # (in place with another stride)
    for name in ("history", "history_len", "bias", "bias_start", "bias_ids", "mask", "mask_row"):
        assert adjust(**{name: None}) == EINVAL                                                      # one without the other
    for name in ("history", "history_len", "prompt_len", "repetition", "presence", "frequency", "bias_start", "bias_ids", "bias", "mask", "mask_row"):
        assert adjust(**{name: 4098}) == EINVAL
    assert adjust(history_stride=-1) == EINVAL and adjust(history_stride=(1 << 30) + 1) == ELIMIT
    assert adjust(n_bias=-1) == EINVAL and adjust(n_bias=2 ** 31 - 1) == EINVAL and adjust(n_masks=-1) == EINVAL and adjust(mask_stride=31) == EINVAL


@pytest.mark.parametrize("mask", [4096, None])
def test_no_rows_have_no_tensors(mask):
    """What has no elements has no address, either: a call of no rows takes NULL for all that has a number a row."""
    assert adjust(n=0, z=None, out=None, ids=None, mask=mask, mask_row=None) == 0
    assert adjust(n=0, z=None, out=None, ids=None, mask=mask, mask_row=None, zs=0, outs=0) == 0
    assert adjust(n=1, z=None, mask=mask, mask_row=None) == EINVAL and adjust(n=1, out=None, mask=mask, mask_row=mask) == EINVAL
    for kw in (dict(rules=False), dict(start=None), dict(seqs=0), dict(vocab=0), dict(dtype=3), dict(history=None), dict(bias_ids=None), dict(n_bias=-1), dict(z=ctypes.c_void_p(4097))):
        assert adjust(n=0, **kw) == EINVAL                                                           # (what is wrong with rows or without)


def test_binding_refuses_what_the_library_cannot_see():
    t, i32, u8 = torch.zeros, torch.int32, torch.uint8
    codes, scales = t(3, 16, 4, 32, dtype=u8), t(3, 16, 4, 2, dtype=u8)
    place = (t(1, 3, dtype=i32), t(2, dtype=i32), t(1, dtype=i32))
    with pytest.raises(ValueError):           # not on a GPU
        binding.ppd_paged_attention_fp4(t(2, 4, 64), codes, scales, codes, scales, *place)
    with pytest.raises(ValueError):
        binding.ppd_paged_plan(place[0], t(3, dtype=i32), t(2, dtype=torch.int64), place[2], place[2], 16, 1)
    with pytest.raises(ValueError):
        binding.ppd_adjust_logits(t(2, 50), place[1])
    binding._paged_args_fp4(codes, scales, codes, scales, *place, torch.float32, 2)
    other = t(3, 16, 4, 64, dtype=u8)[..., ::2]
    for bad in ((codes, scales, codes[:2], scales), (codes, scales, codes, scales[:2]), (codes.char(), scales, codes, scales), (codes, scales.int(), codes, scales),
                (codes, codes, codes, codes), (other, scales, other, scales), (codes[0], scales[0], codes[0], scales[0])):
        with pytest.raises(ValueError):
            binding._paged_args_fp4(*bad, *place, torch.float32, 2)
    with pytest.raises(ValueError):
        binding._paged_args_fp4(codes, scales, codes, scales, *place, torch.float64, 2)
    with pytest.raises(ValueError):
        binding._paged_args_fp4(codes, scales, codes, scales, place[0], t(3, dtype=i32), place[2], torch.float32, 2)
