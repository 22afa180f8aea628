"""What the serving operators refuse or ask for at the ends of their ranges: host logic only, no kernel is launched."""
import ctypes as C

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
