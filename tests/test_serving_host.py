"""Refusals and sizes of the serving operators: host logic only, no kernel is launched and no device memory touched."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_07306_amd import binding as PB
from tests import serving_reference as R

BAD, NULL, SMALL = PB.PT_ERR_INVALID_ARGUMENT, PB.PT_ERR_NULL_POINTER, PB.PT_ERR_ARENA_TOO_SMALL


def cache(**kw):
    d = dict(k=0x10000, v=0x20000, dtype=PB.PT_BF16, n_layers=2, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64,
             layer_stride=20480, page_stride=2048, head_stride=1024, token_stride=64)
    d.update(kw)
    return PB.pt_paged_cache(*[d[n] for n, _ in PB.pt_paged_cache._fields_])


def batch(**kw):
    d = dict(row_start=0x1000, kv_len=0x2000, pages=0x3000, pages_stride=8, n_seqs=3, total_rows=5, max_q_len=0, max_kv_len=0, status=None)
    d.update(kw)
    return PB.pt_paged_batch(*[d[n] for n, _ in PB.pt_paged_batch._fields_])


def rows(data=0x40000, row_stride=256, head_stride=64):
    return PB.pt_head_rows(data, row_stride, head_stride)


CACHE_FAULTS = [dict(dtype=2), dict(n_layers=0), dict(n_pages=0), dict(n_kv_heads=0), dict(page_size=0), dict(page_size=8), dict(page_size=48), dict(page_size=8192),
                dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(k=0x10008), dict(v=0x20002), dict(layer_stride=-8), dict(page_stride=-8),
                dict(head_stride=4), dict(token_stride=56), dict(token_stride=68), dict(token_stride=(1 << 24) + 8), dict(page_stride=2044),
                dict(dtype=PB.PT_F32, token_stride=66), dict(page_size=4096, token_stride=1 << 19)]
BATCH_FAULTS = [dict(n_seqs=-1), dict(total_rows=-1), dict(pages_stride=-1), dict(max_q_len=-1), dict(max_kv_len=-1), dict(max_kv_len=129),
                dict(row_start=0x1002), dict(kv_len=0x2001), dict(pages=0x3003), dict(status=0x5001)]


def attend(c=None, layer=0, b=None, q=None, o=None, heads=4, scale=0.125, causal=1, ws=0x100000, size=1 << 30):
    c, b = c or cache(), b or batch()
    return PB.lib().pt_paged_attention(c, layer, b, q or rows(), o or rows(0x80000), heads, scale, causal, ws, size, None)


def append(c=None, layer=0, b=None, rope=None, q=None, qo=None, heads=4, k=None, v=None):
    return PB.lib().pt_paged_append(c or cache(), layer, b or batch(), rope, q, qo, heads, k or rows(0x50000), v or rows(0x60000), None)


@pytest.mark.parametrize("fault", CACHE_FAULTS, ids=str)
def test_caches_that_are_refused(fault):
    n = C.c_size_t()
    assert attend(cache(**fault)) == BAD and PB.pt_last_error()
    assert append(cache(**fault)) == BAD
    assert PB.lib().pt_page_copy(cache(**fault), (C.c_int32 * 2)(0, 1), 1, None) == BAD
    assert PB.lib().pt_paged_attention_bytes(cache(**fault), batch(), 4, C.byref(n)) == BAD


@pytest.mark.parametrize("fault", BATCH_FAULTS, ids=str)
def test_batches_that_are_refused(fault):
    assert attend(b=batch(**fault)) == BAD and append(b=batch(**fault)) == BAD


def test_missing_pointers():
    L = PB.lib()
    n = C.c_size_t()
    for fault in (dict(row_start=None), dict(kv_len=None), dict(pages=None)):
        assert attend(b=batch(**fault)) == NULL and append(b=batch(**fault)) == NULL
    for fault in (dict(k=None), dict(v=None)):
        assert attend(cache(**fault)) == NULL and append(cache(**fault)) == NULL
        assert L.pt_page_copy(cache(**fault), (C.c_int32 * 2)(0, 1), 1, None) == NULL
    assert L.pt_paged_attention(None, 0, batch(), rows(), rows(), 4, 1.0, 1, None, 0, None) == NULL
    assert L.pt_paged_attention(cache(), 0, None, rows(), rows(), 4, 1.0, 1, None, 0, None) == NULL
    assert L.pt_paged_attention(cache(), 0, batch(), None, rows(), 4, 1.0, 1, None, 0, None) == NULL
    assert attend(o=rows(None)) == NULL
    assert L.pt_paged_append(cache(), 0, batch(), None, None, None, 0, None, rows(), None) == NULL
    assert L.pt_paged_append(None, 0, batch(), None, None, None, 0, rows(), rows(), None) == NULL
    assert append(q=rows()) == NULL and append(qo=rows()) == NULL
    assert L.pt_page_copy(None, (C.c_int32 * 2)(0, 1), 1, None) == NULL
    assert L.pt_page_copy(cache(), None, 1, None) == NULL
    assert L.pt_paged_attention_bytes(cache(), batch(), 4, None) == NULL
    assert L.pt_sample_bytes(1, 1, None) == NULL
    assert L.pt_rope_init(None, 0, 64, 1e4, 0, 1, 1, 2, 1, 1) == NULL
    assert L.pt_sample(None, 8, 1, 8, 0x100, None, None, None, None, 0x200, None, 0, None) == NULL
    assert L.pt_sample(0x100, 8, 1, 8, None, None, None, None, None, 0x200, None, 0, None) == NULL
    assert L.pt_sample(0x100, 8, 1, 8, 0x100, None, None, None, None, None, None, 0, None) == NULL


def test_operands_that_are_refused():
    for bad in (rows(0x40008), rows(row_stride=-8), rows(row_stride=252), rows(head_stride=12)):
        assert attend(q=bad) == BAD and attend(o=bad) == BAD
        assert append(k=bad) == BAD and append(v=bad) == BAD
        assert append(q=bad, qo=rows()) == BAD and append(q=rows(), qo=bad) == BAD
    for layer in (-1, 2):
        assert attend(layer=layer) == BAD and append(layer=layer) == BAD
    for heads in (0, -4, 3):
        assert attend(heads=heads) == BAD
    assert append(q=rows(), qo=rows(0x90000), heads=0) == BAD
    for scale in (float("nan"), float("inf")):
        assert attend(scale=scale) == BAD
    # the same buffer read and written with other strides
    assert attend(q=rows(), o=rows(row_stride=512)) == BAD
    assert append(q=rows(), qo=rows(head_stride=128)) == BAD


def test_nothing_to_do_is_no_error():
    for b in (batch(n_seqs=0), batch(total_rows=0), batch(n_seqs=0, row_start=None, kv_len=None, pages=None)):
        assert attend(b=b, ws=None, size=0) == 0 and append(b=b) == 0
    L = PB.lib()
    assert L.pt_page_copy(cache(), None, 0, None) == 0
    assert L.pt_sample(None, 0, 0, 8, None, None, None, None, None, None, None, 0, None) == 0
    n = C.c_size_t(5)
    assert L.pt_sample_bytes(0, 8, C.byref(n)) == 0 and n.value == 0


def test_workspace_of_long_sequences():
    c = cache(n_pages=4000)
    b = batch(pages_stride=4096, n_seqs=1, total_rows=1, max_q_len=1, max_kv_len=50000)
    n = C.c_size_t()
    assert PB.lib().pt_paged_attention_bytes(c, b, 4, C.byref(n)) == 0 and 0 < n.value < 1 << 20
    assert attend(c, b=b, ws=None) == NULL
    assert attend(c, b=b, ws=0x100008) == BAD
    assert attend(c, b=b, size=n.value - 1) == SMALL and str(n.value) in PB.pt_last_error()
    # one tile of keys needs none
    assert PB.lib().pt_paged_attention_bytes(c, batch(max_kv_len=64), 4, C.byref(n)) == 0 and n.value == 0


def test_batches_too_large_for_one_launch_are_refused():
    n = C.c_size_t()
    c = cache(n_kv_heads=1, head_stride=0)
    assert PB.lib().pt_paged_attention_bytes(c, batch(n_seqs=2 ** 31 - 1, total_rows=2 ** 31 - 1), 2 ** 10, C.byref(n)) == BAD


def test_calls_whose_launches_would_hold_2_to_the_32_threads_are_refused():
    n = C.c_size_t()
    L = PB.lib()
    assert append(b=batch(total_rows=(1 << 23) + 1)) == BAD and "2^23" in PB.pt_last_error()
    assert attend(b=batch(total_rows=(1 << 23) + 1)) == BAD
    # 2^20 rows of 16 heads on one KV head: 2^20 tiles of 16 rows; long ones are joined row by row
    c = cache(dtype=PB.PT_F32, n_kv_heads=1, n_pages=100000, head_stride=0)
    assert L.pt_paged_attention_bytes(c, batch(total_rows=1 << 20, n_seqs=1, pages_stride=512, max_kv_len=8192), 16, C.byref(n)) == 0
    assert L.pt_paged_attention_bytes(c, batch(total_rows=1 << 20, n_seqs=1, pages_stride=1024, max_kv_len=16384), 16, C.byref(n)) == BAD
    assert "too many tiles" in PB.pt_last_error()
    assert L.pt_sample_bytes(1 << 21, 100, C.byref(n)) == 0 and L.pt_sample_bytes((1 << 21) + 1, 100, C.byref(n)) == BAD
    assert L.pt_sample(0x1000, 100, (1 << 21) + 1, 100, 0x2000, None, None, None, None, 0x3000, None, 0, None) == BAD


@pytest.mark.parametrize("args", [(2, 64, 1e4, 0, 1, 1, 2, 1, 1), (-1, 64, 1e4, 0, 1, 1, 2, 1, 1), (0, 0, 1e4, 0, 1, 1, 2, 1, 1), (0, 63, 1e4, 0, 1, 1, 2, 1, 1),
                                  (0, 258, 1e4, 0, 1, 1, 2, 1, 1), (0, 64, 0.0, 0, 1, 1, 2, 1, 1), (0, 64, float("nan"), 0, 1, 1, 2, 1, 1),
                                  (0, 64, float("inf"), 0, 1, 1, 2, 1, 1), (0, 64, 1e4, 3, 1, 1, 2, 1, 1), (0, 64, 1e4, 1, 0.0, 1, 2, 1, 1),
                                  (0, 64, 1e4, 1, float("inf"), 1, 2, 1, 1), (0, 64, 1e4, 2, 4, 2, 2, 1, 1), (0, 64, 1e4, 2, 4, -1, 2, 1, 1),
                                  (0, 64, 1e4, 2, 4, 1, 2, 0, 1), (0, 64, 1e4, 0, 1, 1, 2, 1, float("nan"))])
def test_rotary_descriptions_that_are_refused(args):
    assert PB.lib().pt_rope_init(C.byref(PB.pt_rope()), *args) == BAD


def test_rotary_frequencies():
    for scaling, code, kw in (("none", 0, {}), ("linear", 1, dict(factor=8.0)), ("by_parts", 2, dict(factor=16.0, low=1.0, high=32.0, original_len=4096))):
        r = PB.PTRope(PB.PT_ROPE_HALF, 128, 500000.0, scaling=code, **kw)
        f = R.frequencies(128, 500000.0, scaling, **kw) / (2 * np.pi)
        assert np.max(np.abs(np.array(r.c.turns)[:64] / f - 1)) < 1e-14
    # by parts: the fast pairs keep their frequency, the slow ones are divided, nothing lies outside
    plain, parts = R.frequencies(128, 500000.0, "none"), np.array(r.c.turns)[:64] * 2 * np.pi
    assert np.allclose(parts[0], plain[0], rtol=1e-14) and np.allclose(parts[-1], plain[-1] / 16, rtol=1e-14)
    assert np.all(parts <= plain * (1 + 1e-14)) and np.all(parts >= plain / 16 * (1 - 1e-14))


def test_a_rotation_wider_than_the_head_is_refused():
    r = PB.PTRope(PB.PT_ROPE_HALF, 128)
    assert append(rope=r.c) == BAD
    assert append(rope=PB.pt_rope()) == BAD           # not filled by pt_rope_init


def copy(pairs, **kw):
    flat = [x for p in pairs for x in p]
    return PB.lib().pt_page_copy(cache(**kw), (C.c_int32 * len(flat))(*flat), len(pairs), None)


def test_page_copies_that_are_refused():
    for many in (10, 100000):       # both forms of the check
        assert copy([(0, many)], n_pages=many) == BAD and "names page" in PB.pt_last_error()
        assert copy([(-1, 2)], n_pages=many) == BAD and copy([(many, 2)], n_pages=many) == BAD and copy([(1, -1)], n_pages=many) == BAD
        assert copy([(0, 2), (1, 2)], n_pages=many) == BAD and "twice" in PB.pt_last_error()
        assert copy([(0, 1), (1, 2)], n_pages=many) == BAD and "both" in PB.pt_last_error()
        assert copy([(5, 5)], n_pages=many) == BAD
    assert PB.lib().pt_page_copy(cache(), (C.c_int32 * 2)(0, 1), -1, None) == BAD


def test_sampling_calls_that_are_refused():
    L = PB.lib()
    ok = [0x100, 8, 2, 8, 0x200, None, None, None, None, 0x300, None, 0, None]
    for at, value in ((2, -1), (3, 0), (3, (1 << 24) + 1), (1, 7), (1, -1), (0, 0x102), (4, 0x201), (5, 0x1), (6, 0x2), (7, 0x3), (8, 0x5), (9, 0x301)):
        args = list(ok)
        args[at] = value
        assert L.pt_sample(*args) == BAD, (at, value)


def test_binding_checks():
    torch = pytest.importorskip("torch")
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    good = t(1, 4, 2, 16, 64)
    for k, v in ((good[0], good[0]), (good, t(1, 4, 2, 16, 32)), (good, good.bfloat16()), (good.half(), good.half()), (good, t(1, 4, 16, 2, 64).transpose(2, 3)),
                 (t(1, 4, 2, 64, 16).transpose(3, 4), t(1, 4, 2, 64, 16).transpose(3, 4))):
        with pytest.raises(PB.PTError):
            PB.PTPagedCache(k, v)
    for args in ((i32(3), i32(3), i32(3, 4)), (i32(4), i32(3), i32(2, 4)), (i32(4).long(), i32(3), i32(3, 4)), (i32(4), i32(3), i32(4, 3).t()),
                 (i32(8)[::2], i32(3), i32(3, 4)), (i32(4), i32(3), i32(4).expand(3, 4))):
        with pytest.raises(PB.PTError):
            PB.PTPagedBatch(*args, total_rows=3)
    c = PB.PTPagedCache(good, good.clone())
    b = PB.PTPagedBatch(i32(4), i32(3), i32(3, 4), total_rows=3)
    assert b.bound(c).max_kv_len == 64
    with pytest.raises(PB.PTError):
        PB.PTPagedBatch(i32(4), i32(3), i32(3, 4), total_rows=3, max_kv_len=65).bound(c)
    for q in (t(2, 4, 64), t(3, 4, 32), t(3, 4, 64).bfloat16(), t(3, 256), t(3, 4, 128)[..., ::2]):
        with pytest.raises(PB.PTError):
            PB.pt_paged_attention(c, 0, b, q)
    with pytest.raises(PB.PTError):
        PB.pt_paged_attention(c, 0, b, t(3, 4, 64))           # host memory
    with pytest.raises(PB.PTError):
        PB.pt_paged_append(c, 0, b, t(3, 1, 64), t(3, 2, 64))  # too few heads
    for pairs in ([0, 1], [[0, 1, 2]], [[0.5, 1.0]], np.array([[0, 2 ** 32 + 1]])):
        with pytest.raises(PB.PTError):
            PB.pt_page_copy(c, pairs)
    for kw in (dict(uniform=t(3)), dict(uniform=t(2).double()), dict(uniform=t(2), top_k=t(2)), dict(uniform=t(2), top_p=t(2, 1)), dict(uniform=t(4)[::2])):
        with pytest.raises(PB.PTError):
            PB.pt_sample(t(2, 8), **kw)
    with pytest.raises(PB.PTError):
        PB.pt_sample(t(8, 2).t(), t(2))
