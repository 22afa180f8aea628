"""What the serving operators refuse or ask for at the ends of their ranges: host logic only, no kernel is launched."""
import ctypes as C

import pytest

from paper_2602_07306_amd import binding as PB
from tests.test_serving_host import BAD, batch, cache


def attention_bytes(c, b, heads):
    n = C.c_size_t()
    rc = PB.lib().pt_paged_attention_bytes(c, b, heads, C.byref(n))
    return rc, n.value


def test_workgroups_of_both_kinds_in_one_launch_are_counted_in_whole_stretches():
    """A launch of both kinds rounds each kind's workgroups up to stretches of 64, and holds less than 2^24 of 256 threads.
    16 heads on one KV head, up to three rows a sequence: a workgroup per sequence for those of one row, and one for each
    that may have 17 packed rows or more."""
    many = 1 + 64 * 100000                       # rows * 16 / 17 such sequences
    rows = (many * 17 + 15) // 16
    assert rows <= 1 << 23 and rows * 16 // 17 == many
    b = lambda few: batch(n_seqs=few, total_rows=rows, max_q_len=3, max_kv_len=100)
    c = cache(n_kv_heads=1, head_stride=0)
    few = (1 << 24) - 126 - many                 # 2^24 with both rounded up
    assert few % 64 == 1
    assert attention_bytes(c, b(few), 16)[0] == BAD and "too many tiles" in PB.pt_last_error()
    assert attention_bytes(c, b(few - 1), 16) == (0, 0)


def test_workspaces_hold_the_partials_of_rows_that_are_cut_and_no_others():
    """A partial is head_dim + 2 fp32 values per head of a row and range, 64 ranges at most.  Sequences of few rows: 16 packed
    rows each, of as many heads as share a KV head.  Chunks of more tiles than fill the chip are not cut."""
    c = lambda **kw: cache(n_kv_heads=8, head_dim=128, page_size=32, n_pages=100000, token_stride=128, head_stride=4096, page_stride=32768, layer_stride=0, **kw)
    part, group = 4 * 130 * 64, 8                # bytes of a row's partials in one range, 64 heads
    few = lambda n: n * (16 // group) * part * 64 + 32
    for seqs, rows, longest in ((2, 2049, 16384), (2, 2049, 131072), (8, 8199, 131072), (40, 36 + 4 * 400, 2048)):
        rc, n = attention_bytes(c(), batch(n_seqs=seqs, total_rows=rows, pages_stride=8192, max_q_len=rows - seqs + 1, max_kv_len=longest), 64)
        assert rc == 0 and 0 < n <= few(seqs), (seqs, rows, longest, n)
    assert attention_bytes(c(), batch(n_seqs=2, total_rows=4096, pages_stride=8192, max_q_len=2048, max_kv_len=16384), 64)[1] <= few(2)
    assert attention_bytes(c(), batch(n_seqs=1, total_rows=2048, pages_stride=8192, max_q_len=2048, max_kv_len=131072), 64) == (0, 0)
    # one chunk of a few tiles: its ranges make up 512 workgroups, a range for each of them and one more round
    rc, n = attention_bytes(c(), batch(n_seqs=1, total_rows=300, pages_stride=8192, max_q_len=300, max_kv_len=131072), 64)
    assert rc == 0 and 0 < n <= (512 + 160) * 128 * 4 * 130 + 32
    # decode steps alone: by rows, as many as there are
    rc, n = attention_bytes(c(), batch(n_seqs=16, total_rows=16, pages_stride=8192, max_q_len=1, max_kv_len=131072), 64)
    assert rc == 0 and n == 16 * 16 * part


def test_buffers_of_no_rows_may_have_no_address():
    """An empty tensor has none; there is nothing to do with it."""
    L, none = PB.lib(), PB.pt_head_rows(None, 256, 64)
    for b in (batch(total_rows=0), batch(n_seqs=0), batch(n_seqs=0, total_rows=0, row_start=None, kv_len=None, pages=None, pages_stride=0)):
        assert L.pt_paged_attention(cache(), 0, b, none, none, 4, 0.125, 1, None, 0, None) == 0
        assert L.pt_paged_append(cache(), 0, b, None, none, none, 4, none, none, None) == 0
        other = PB.pt_head_rows(None, 512, 128)               # not the same buffer
        assert L.pt_paged_attention(cache(), 0, b, none, other, 4, 0.125, 1, None, 0, None) == 0
        assert L.pt_paged_append(cache(), 0, b, None, none, other, 4, none, none, None) == 0
        # the descriptors themselves are asked for all the same, and what they say has to make sense
        assert L.pt_paged_attention(cache(), 0, b, None, none, 4, 0.125, 1, None, 0, None) == PB.PT_ERR_NULL_POINTER
        assert L.pt_paged_attention(cache(), 0, b, PB.pt_head_rows(None, 252, 64), none, 4, 0.125, 1, None, 0, None) == BAD
    assert L.pt_paged_attention(cache(), 0, batch(), none, none, 4, 0.125, 1, None, 0, None) == PB.PT_ERR_NULL_POINTER


def test_a_batch_used_with_two_caches_keeps_a_descriptor_for_each():
    """The bound that follows from the table's width and the page size belongs to the call, not to the batch."""
    torch = pytest.importorskip("torch")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    small, large = (PB.PTPagedCache(*(torch.zeros((1, 4, 2, page, 64)) for _ in range(2))) for page in (16, 64))
    b = PB.PTPagedBatch(i32(4), i32(3), i32(3, 4), total_rows=3)
    first = b.bound(small)
    second = b.bound(large)
    assert (first.max_kv_len, second.max_kv_len, b.bound(small).max_kv_len) == (64, 256, 64)
    given = PB.PTPagedBatch(i32(4), i32(3), i32(3, 4), total_rows=3, max_kv_len=100)
    assert given.bound(large).max_kv_len == 100
    with pytest.raises(PB.PTError):
        given.bound(small)


def test_append_refuses_more_heads_than_its_numbers_hold():
    rows = lambda at: PB.pt_head_rows(at, 256, 64)
    append = lambda heads, **kw: PB.lib().pt_paged_append(cache(**kw), 0, batch(), None, rows(0x40000), rows(0x80000), heads, rows(0x50000), rows(0x60000), None)
    for heads in (2 ** 31 - 1, 2 ** 30 - 1):          # beside 2 KV heads
        assert append(heads) == BAD and "heads" in PB.pt_last_error()
    assert append(4, n_kv_heads=2 ** 31 - 1) == BAD
