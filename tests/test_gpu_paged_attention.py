"""pt_paged_attention against a plain 64-bit attention: head layouts, lengths from nothing to thousands, chunks, pages that end
inside tiles, strides, masks, values that are no numbers, pools past 32 bits, graphs and streams."""
import numpy as np
import pytest

from tests import serving_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Problem:
    """A batch with its pool: lens = [(new rows, positions)], everything that no row may see filled with NaN."""

    def __init__(self, H, Hkv, hd, dtype, page, lens, seed=0, layers=2, layer=1, order="head", tail_rows=3, scale_q=1.0):
        from paper_2602_07306_amd import binding as PB
        self.PB, self.layer, self.page, self.hd, self.lens = PB, layer, page, hd, lens
        rng = np.random.default_rng(seed)
        ty = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.bf16 = dtype == "bf16"
        self.row_start = np.concatenate([[0], np.cumsum([n for n, _ in lens])]).astype(np.int32)
        self.kv_len = np.array([k for _, k in lens], dtype=np.int32)
        self.table, total = R.page_table(rng, self.kv_len, page)
        self.rows = int(self.row_start[-1]) + tail_rows
        gen = torch.Generator().manual_seed(seed)
        k = torch.full((total, Hkv, page, hd), float("nan"))
        v = k.clone()
        for b, n in enumerate(self.kv_len):
            for p in range(0, n, page):
                m = min(page, n - p)
                k[self.table[b, p // page], :, :m] = torch.randn((Hkv, m, hd), generator=gen)
                v[self.table[b, p // page], :, :m] = torch.randn((Hkv, m, hd), generator=gen)
        shape = (layers, total, Hkv, page, hd) if order == "head" else (layers, total, page, Hkv, hd)
        self.k5, self.v5 = (torch.full(shape, float("nan"), dtype=ty, device="cuda") for _ in range(2))
        if order == "token":
            self.k5, self.v5 = self.k5.transpose(2, 3), self.v5.transpose(2, 3)
        self.k5[layer], self.v5[layer] = k.to(ty).cuda(), v.to(ty).cuda()
        # queries inside a wider buffer, as a fused product leaves them
        wide = torch.randn((self.rows, H + 2 * Hkv, hd), generator=gen) * scale_q
        self.q = wide.to(ty).cuda()[:, :H]
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.cache = PB.PTPagedCache(self.k5, self.v5)
        self.batch = self.make_batch(max_q_len=max(n for n, _ in lens), max_kv_len=max(1, int(self.kv_len.max())))

    def make_batch(self, **kw):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        return self.PB.PTPagedBatch(dev(self.row_start), dev(self.kv_len), dev(self.table), total_rows=self.rows, status=self.status, **kw)

    def run(self, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        self.PB.pt_paged_attention(self.cache, self.layer, self.batch, self.q, out=out, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, out, scale=None, causal=True, rows=None):
        scale = self.hd ** -0.5 if scale is None else scale
        ref, weight, score = R.attention(R.f64(self.q), R.f64(self.k5[self.layer]), R.f64(self.v5[self.layer]), self.table, self.row_start, self.kv_len,
                                         self.page, scale, causal)
        tol = R.attention_bound(ref, weight, score, self.hd, int(self.kv_len.max()), self.bf16)
        got = R.f64(out)
        used = int(self.row_start[-1])
        assert np.all(got[used:] == 7.0)                     # rows behind the last sequence
        sel = slice(0, used) if rows is None else rows
        bad = ~(np.abs(got[sel] - ref[sel]) <= tol[sel])
        assert not bad.any(), "%d values off, worst %.3g times its bound" % (bad.sum(), np.nanmax(np.abs(got[sel] - ref[sel]) / tol[sel]))


MIXED = [(5, 5), (1, 300), (0, 40), (33, 100), (64, 64), (3, 2), (0, 0), (1, 1), (17, 65)]
SHAPES = [(4, 4, 64, "bf16", 16), (8, 2, 128, "bf16", 32), (16, 1, 128, "bf16", 64), (24, 1, 64, "bf16", 16), (6, 2, 80, "bf16", 16), (2, 2, 256, "bf16", 16),
          (4, 1, 192, "bf16", 128), (2, 1, 8, "bf16", 16), (4, 2, 32, "fp32", 16), (4, 4, 128, "fp32", 64), (2, 2, 256, "fp32", 16), (3, 1, 72, "fp32", 32),
          (40, 1, 16, "fp32", 16)]


@pytest.mark.parametrize("H,Hkv,hd,dtype,page", SHAPES)
@pytest.mark.parametrize("lens", [[(1, 1)], [(1, 777), (1, 16), (1, 17), (1, 64), (1, 1)], MIXED, [(130, 700), (1, 5)]], ids=["one", "decode", "mixed", "chunk"])
def test_against_the_definition(H, Hkv, hd, dtype, page, lens):
    p = Problem(H, Hkv, hd, dtype, page, lens, seed=H + hd)
    p.check(p.run())
    assert int(p.status) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens", [[(1, 50), (1, 1)], MIXED])
def test_without_a_mask(dtype, lens):
    p = Problem(4, 2, 64, dtype, 16, lens, seed=3)
    p.check(p.run(causal=False), causal=False)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("order", ["head", "token"])
def test_pages_in_either_order(dtype, hd, order):
    p = Problem(4, 2, hd, dtype, 32, MIXED, seed=4, order=order)
    p.check(p.run())


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-3])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scales(dtype, scale):
    p = Problem(4, 2, 64, dtype, 16, [(1, 200), (9, 40)], seed=5)
    p.check(p.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores_do_not_overflow(dtype):
    p = Problem(4, 2, 64, dtype, 16, [(1, 200), (9, 40)], seed=6)
    p.q.mul_(300.0)          # scores of several thousand: the running maximum moves far
    # a score's error of 2^-24 of its terms' sum is no longer small against 1, so the bound is useless: one key wins instead
    out = p.run()
    assert torch.isfinite(out[:10].float()).all()


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_later_position_has_no_influence(dtype, hd, bad):
    """The last keys of a chunk are no numbers: rows before them are as if they were not there, rows that see them are not."""
    lens = [(40, 40), (150, 400), (2, 30)]
    p = Problem(4, 2, hd, dtype, 16, lens, seed=7)
    clean = p.run()
    for b, (n, kv) in enumerate(lens):
        for pos in (kv - 1, kv - n // 2):
            p.k5[p.layer, p.table[b, pos // 16], :, pos % 16] = bad
            p.v5[p.layer, p.table[b, pos // 16], :, pos % 16] = bad
    out = p.run()
    for b, (n, kv) in enumerate(lens):
        first = int(p.row_start[b])
        good = n - max(1, n // 2)          # rows before the first bad key
        p_rows = slice(first, first + good)
        ref = clean[p_rows].float()
        assert torch.isfinite(out[p_rows].float()).all()
        # the rows' own keys are as before: both are within the bound of one truth
        r, w, s = R.attention(R.f64(p.q), np.nan_to_num(R.f64(p.k5[p.layer]), nan=0, posinf=0, neginf=0),
                              np.nan_to_num(R.f64(p.v5[p.layer]), nan=0, posinf=0, neginf=0), p.table, p.row_start, p.kv_len, 16, hd ** -0.5)
        tol = R.attention_bound(r, w, s, hd, kv, p.bf16)
        assert np.all(np.abs(R.f64(out[p_rows]) - r[p_rows]) <= tol[p_rows])
        assert np.all(np.abs(R.f64(ref) - r[p_rows]) <= tol[p_rows])
        assert not torch.isfinite(out[first + n - 1].float()).all()


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_a_visible_position_has_all_its_influence(dtype, hd):
    """No number among the keys that every row sees: every row is none, and nothing is taken for a key behind it."""
    lens = [(40, 140), (150, 400), (1, 30)]
    p = Problem(4, 2, hd, dtype, 16, lens, seed=19)
    for b in range(3):
        p.v5[p.layer, p.table[b, 0], :, 3, 5] = float("inf")
    out = p.run()
    used = int(p.row_start[-1])
    assert torch.all(out[:used, :, 5] == float("inf"))
    keep = [c for c in range(hd) if c != 5]
    p.v5[p.layer, p.table[[0, 1, 2], 0], :, 3, 5] = 0
    assert torch.equal(out[:used][..., keep], p.run()[:used][..., keep])


@pytest.mark.parametrize("H,Hkv,hd,dtype", [(2, 2, 128, "bf16"), (8, 1, 64, "bf16"), (2, 1, 64, "fp32")])
def test_long_sequences_cut_into_ranges(H, Hkv, hd, dtype):
    p = Problem(H, Hkv, hd, dtype, 64, [(1, 5003), (1, 130), (3, 2049), (1, 1)], seed=8)
    assert p.PB.pt_paged_attention_bytes(p.cache, p.batch, H) > 0
    a = p.run()
    p.check(a)
    assert torch.equal(a, p.run())       # the same from call to call


@pytest.mark.parametrize("H,hd,dtype", [(1, 128, "bf16"), (20, 128, "bf16"), (2, 96, "bf16"), (1, 64, "bf16"), (3, 256, "bf16"), (2, 64, "fp32")])
def test_very_long_sequences(H, hd, dtype):
    # ranges of more than 1024 keys, more than 50 of them, beside sequences of one range and of two
    p = Problem(H, 1, hd, dtype, 64, [(1, 70001), (1, 30), (1, 1025), (0, 0), (1, 1300)], seed=H + hd, layers=1, layer=0)
    out = p.run()
    p.check(out)
    assert torch.equal(p.run(), out)


def test_bounds_need_not_be_tight():
    p = Problem(4, 2, 64, "bf16", 16, MIXED, seed=9)
    tight = p.run()
    p.batch = p.make_batch()             # nothing but the buffers' sizes known
    out = p.run()
    p.check(out)
    p.check(tight)


def test_many_sequences():
    rng = np.random.default_rng(10)
    lens = [(int(rng.integers(0, 4)), int(rng.integers(4, 60))) for _ in range(300)]
    p = Problem(4, 2, 64, "bf16", 16, lens, seed=10)
    p.check(p.run())
    lens = [(int(n > 2), k) for n, k in lens]
    p = Problem(2, 2, 64, "fp32", 16, lens, seed=11)
    p.check(p.run())


def test_in_place():
    p = Problem(4, 2, 64, "bf16", 16, MIXED, seed=12)
    want = p.run()
    keep = p.q.clone()
    p.PB.pt_paged_attention(p.cache, p.layer, p.batch, p.q, out=p.q)
    used = int(p.row_start[-1])
    assert torch.equal(p.q[:used], want[:used]) and torch.equal(p.q[used:], keep[used:])


@pytest.mark.parametrize("G", [1, 4])
def test_in_place_before_a_position_that_is_no_number(G):
    """The rows in front of it are computed anew from their queries, which lie where the output goes."""
    p = Problem(2 * G, 2, 64, "bf16", 16, [(60, 90), (1, 30), (3, 20)], seed=20)
    for b in (0, 2):
        last = int(p.kv_len[b]) - 1
        p.v5[p.layer, p.table[b, last // 16], :, last % 16] = float("nan")
    want = p.run()
    used = int(p.row_start[-1])
    p.PB.pt_paged_attention(p.cache, p.layer, p.batch, p.q, out=p.q)
    got = p.q[:used].float()
    assert torch.equal(torch.isnan(got), torch.isnan(want[:used].float())) and not torch.isnan(got[:59]).any()
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want[:used].float()))


def test_pages_that_do_not_exist_are_reported():
    p = Problem(4, 2, 64, "bf16", 16, [(1, 40), (1, 40)], seed=13)
    want = p.run()
    p.k5[p.layer, 0] = 0                      # read in the bad page's place
    p.v5[p.layer, 0] = 0
    ok = 0 if 0 in p.table[1] else 1          # a sequence that does not own page 0
    p.table[1 - ok, 1] = 10 ** 6
    p.batch = p.make_batch(max_q_len=1, max_kv_len=40)
    out = p.run()
    assert int(p.status) == 1
    if ok not in (b for b in range(2) if 0 in p.table[b]):
        assert torch.equal(out[ok], want[ok])


def test_contradictory_lengths_are_clamped_and_reported():
    p = Problem(4, 2, 64, "bf16", 16, [(4, 40), (4, 40)], seed=14)
    want = p.run()
    p.kv_len[1] = 10 ** 9
    p.batch = p.make_batch(max_q_len=4, max_kv_len=40)
    out = p.run()
    assert int(p.status) == 2 and torch.equal(out[:4], want[:4])
    p.status.zero_()
    p.kv_len[1] = 40
    p.row_start[:] = [0, 4, 10 ** 9]
    p.batch = p.make_batch(max_q_len=4, max_kv_len=40)
    out = p.run()
    assert int(p.status) == 2 and torch.equal(out[:4], want[:4])


def test_a_pool_past_32_bits():
    """Pages whose elements lie more than 2^32 bytes, and 2^31 elements, from the pool's start."""
    from paper_2602_07306_amd import binding as PB
    pages = (1 << 31) // (2 * 128 * 128) + 40
    k = torch.empty((1, pages, 2, 128, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    p = Problem(4, 2, 128, "bf16", 128, [(1, 1000), (3, 300)], seed=15)
    total = p.k5.shape[1]
    k[0, pages - total:], v[0, pages - total:] = p.k5[p.layer], p.v5[p.layer]
    want = p.run()
    p.table = np.where(p.table >= 0, p.table + (pages - total), p.table).astype(np.int32)
    p.cache = PB.PTPagedCache(k, v)
    p.layer = 0
    p.batch = p.make_batch(max_q_len=3, max_kv_len=1000)
    assert torch.equal(p.run(), want)


def test_captured_graph_follows_its_arrays():
    """A decode step captured once and replayed while the sequences grow."""
    p = Problem(4, 2, 64, "bf16", 16, [(1, 600), (1, 90), (1, 10)], seed=16)
    full = p.kv_len.copy()
    ws = torch.empty(p.PB.pt_paged_attention_bytes(p.cache, p.batch, 4), dtype=torch.uint8, device="cuda")
    out = torch.full(p.q.shape, 7.0, dtype=p.q.dtype, device="cuda")
    call = lambda: p.PB.pt_paged_attention(p.cache, p.layer, p.batch, p.q, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for cut in (0, 5, 9, 3):
        p.kv_len = (full - cut).astype(np.int32)
        p.batch.kv_len.copy_(torch.from_numpy(p.kv_len))
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        p.check(got)
        assert torch.equal(got, p.run())


def test_on_another_stream():
    p = Problem(4, 2, 64, "bf16", 16, MIXED + [(1, 3000)], seed=17)
    want = p.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [p.PB.pt_paged_attention(p.cache, p.layer, p.batch, p.q, stream=side) for _ in range(3)]
    side.synchronize()
    used = int(p.row_start[-1])
    assert all(torch.equal(o[:used], want[:used]) for o in outs)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_an_empty_batch_and_one_sequence_without_rows(dtype):
    p = Problem(2, 2, 64, dtype, 16, [(0, 33), (0, 0)], seed=18)
    assert torch.all(p.run() == 7.0)
    p.batch = p.PB.PTPagedBatch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                                torch.zeros((0, 4), dtype=torch.int32, device="cuda"), total_rows=3)
    assert torch.all(p.run() == 7.0)
