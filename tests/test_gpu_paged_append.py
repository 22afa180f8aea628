"""pt_paged_append against rotation in 64 bits: layouts, parts of the head, scalings, far positions, padding, strides."""
import numpy as np
import pytest

from tests import serving_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LENS = [(1, 1), (5, 20), (0, 9), (3, 2), (17, 100), (1, 64)]      # the fourth begins with a row of padding


def run(H, Hkv, hd, dtype, page, lens, rope=None, kw=None, order="head", q="new", seed=0, past=0):
    """Returns nothing: checks queries, keys, values and everything that must not change."""
    from paper_2602_07306_amd import binding as PB
    ty = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = [(n, kv + past) for n, kv in lens]
    row_start = np.concatenate([[0], np.cumsum([n for n, _ in lens])]).astype(np.int32)
    kv_len = np.array([kv for _, kv in lens], dtype=np.int32)
    first = [max(0, kv - n) // page for n, kv in lens]            # the past needs no pages of its own here
    new, total = R.page_table(rng, [kv - f * page for (_, kv), f in zip(lens, first)], page)
    table = np.full((len(lens), max(f + new.shape[1] for f in first)), -5, dtype=np.int32)
    for b, f in enumerate(first):
        table[b, f:f + new.shape[1]] = new[b]
    rows = int(row_start[-1]) + 2
    shape = (2, total, Hkv, page, hd) if order == "head" else (2, total, page, Hkv, hd)
    k5, v5 = (torch.randn(shape, generator=gen, device="cuda").to(ty) for _ in range(2))
    if order == "token":
        k5, v5 = k5.transpose(2, 3), v5.transpose(2, 3)
    before = k5.clone(), v5.clone()
    qkv = torch.randn((rows, H + 2 * Hkv, hd), generator=gen, device="cuda").to(ty)
    qs, ks, vs = qkv.split((H, Hkv, Hkv), dim=1)
    q_in = R.f64(qs)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()
    batch = PB.PTPagedBatch(dev(row_start), dev(kv_len), dev(table), total_rows=rows, status=status)
    out = None if q is None else qs if q == "same" else torch.full((rows, H, hd), 7.0, dtype=ty, device="cuda")
    PB.pt_paged_append(PB.PTPagedCache(k5, v5), 1, batch, ks, vs, q=None if q is None else qs, q_out=out, rope=rope)
    torch.cuda.synchronize()
    assert int(status) == 0
    used, pos = int(row_start[-1]), R.positions(row_start, kv_len)
    step = R.BF16_STEP if dtype == "bf16" else R.FP32_STEP
    if rope is None:
        turned = lambda x: x
    else:
        freq = R.frequencies(rope.c.rotary_dim, **kw["freq"])
        turned = lambda x: R.rotate(x, pos, freq, kw["layout"], kw.get("magnitude", 1.0))
    # One rounding of the result; before it, in fp32: sine and cosine to 2^-22 of the unit circle (the angle's rest in a
    # float, three roundings of the series, the magnitude), two products and a sum; at most eight steps of the pair's length.
    # The angle itself: 2^-52 of p f_j / 2 pi turns, counted for both sides.
    far = 2 * np.pi * 2.0 ** -51 * (np.abs(pos).max() + 1) * (1 if rope is None else max(1.0, float(np.max(freq))))

    def close(got, ref, x):
        length = np.sqrt((x ** 2).sum(-1, keepdims=True))   # no pair is longer than its head
        tol = np.abs(ref) * step + (0 if rope is None else (8 * R.FP32_STEP + far) * abs(kw.get("magnitude", 1.0)) * length)
        assert np.all(np.abs(got - ref) <= tol), np.max(np.abs(got - ref) / np.maximum(tol, 1e-300))

    if q is not None:
        got = R.f64(out)
        close(got[:used], turned(q_in[:used]), q_in[:used])
        assert np.array_equal(got[used:], q_in[used:] if q == "same" else np.full_like(got[used:], 7.0))
    k_ref, v_ref = turned(R.f64(ks)[:used]), R.f64(vs)[:used]
    owner = np.repeat(np.arange(len(lens)), np.diff(row_start))
    untouched_k, untouched_v = before[0], before[1]
    for r in range(used):
        if pos[r] < 0:
            continue
        pg, slot = table[owner[r], pos[r] // page], pos[r] % page
        close(R.f64(k5[1, pg, :, slot]), k_ref[r], R.f64(ks)[r])
        assert np.array_equal(R.f64(v5[1, pg, :, slot]), v_ref[r])
        untouched_k[1, pg, :, slot] = k5[1, pg, :, slot]
        untouched_v[1, pg, :, slot] = v5[1, pg, :, slot]
    assert torch.equal(untouched_k, k5) and torch.equal(untouched_v, v5)     # nothing else was written


def rope_of(layout, dim, theta=10000.0, scaling="none", magnitude=1.0, **s):
    from paper_2602_07306_amd import binding as PB
    code = {"none": PB.PT_ROPE_UNSCALED, "linear": PB.PT_ROPE_LINEAR, "by_parts": PB.PT_ROPE_BY_PARTS}[scaling]
    r = PB.PTRope(PB.PT_ROPE_HALF if layout == "half" else PB.PT_ROPE_INTERLEAVED, dim, theta, scaling=code, magnitude=magnitude, **s)
    return r, {"layout": layout, "magnitude": magnitude, "freq": dict(theta=theta, scaling=scaling, **s)}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("H,Hkv,hd,dim", [(4, 4, 64, 64), (16, 2, 128, 128), (6, 3, 128, 32), (3, 1, 80, 80), (5, 5, 8, 8), (2, 1, 256, 256), (3, 3, 64, 6), (2, 2, 40, 38), (1, 1, 256, 2)])
def test_layouts_and_parts(dtype, layout, H, Hkv, hd, dim):
    rope, kw = rope_of(layout, dim)
    run(H, Hkv, hd, dtype, 16, LENS, rope, kw, seed=hd + dim)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("past", [0, 5000, 1000003])
@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=8.0), dict(scaling="by_parts", factor=16.0, low=1.0, high=32.0, original_len=4096, magnitude=1.25)])
def test_scaled_for_long_contexts(dtype, past, scaling):
    for layout in ("half", "interleaved"):
        rope, kw = rope_of(layout, 64, 500000.0, **scaling)
        run(4, 2, 128, dtype, 64, LENS, rope, kw, seed=past % 97, past=past)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("order", ["head", "token"])
def test_without_rotation_and_without_queries(dtype, order):
    run(4, 2, 64, dtype, 32, LENS, order=order)
    run(4, 2, 64, dtype, 32, LENS, order=order, q=None)
    rope, kw = rope_of("half", 64)
    run(4, 2, 64, dtype, 32, LENS, rope, kw, order=order, q=None)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place(layout):
    rope, kw = rope_of(layout, 32)
    run(4, 2, 64, "bf16", 16, LENS, rope, kw, q="same")


def test_many_rows_and_heads():
    rope, kw = rope_of("half", 128)
    run(64, 8, 128, "bf16", 64, [(700, 700), (1, 3), (400, 1000)] + [(1, 50)] * 100, rope, kw)


def test_pages_that_do_not_exist_receive_nothing():
    from paper_2602_07306_amd import binding as PB
    k5 = torch.zeros((1, 4, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    v5 = torch.zeros_like(k5)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    status = i32([0])
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (-1, 4, 2 ** 31 - 1):
        status.zero_()
        batch = PB.PTPagedBatch(i32([0, 1, 2, 3]), i32([5, 6, 7]), i32([[0], [bad], [2]]), total_rows=3, status=status)
        k5.zero_()
        v5.zero_()
        PB.pt_paged_append(PB.PTPagedCache(k5, v5), 0, batch, x, x)
        torch.cuda.synchronize()
        assert int(status) == 1
        assert float(k5.float().sum()) == 2 * 2 * 64 and float(v5.float().sum()) == 2 * 2 * 64


def test_captured_graph_follows_its_arrays():
    from paper_2602_07306_amd import binding as PB
    rope, kw = rope_of("half", 64)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k5, v5 = (torch.zeros((1, 8, 2, 16, 64), device="cuda") for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    batch = PB.PTPagedBatch(i32([0, 1, 2]), i32([1, 1]), i32([[0, 1, 2], [5, 6, 7]]), total_rows=2, max_q_len=1, max_kv_len=48)
    q, k, v = (torch.randn((2, n, 64), generator=gen, device="cuda") for n in (4, 2, 2))
    out = torch.empty_like(q)
    cache = PB.PTPagedCache(k5, v5)
    call = lambda: PB.pt_paged_append(cache, 0, batch, k, v, q=q, q_out=out, rope=rope)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for n in (3, 17, 40, 18):
        batch.kv_len.fill_(n)
        k.normal_(generator=gen)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), k5.clone(), v5.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], k5) and torch.equal(got[2], v5)
        assert torch.equal(v5[0, 6 if 16 < n <= 32 else 7 if n > 32 else 5, :, (n - 1) % 16], v[1])
