"""pt_sample against the definition in 64 bits, row by row: tokens have to be equal."""
import numpy as np
import pytest

from tests import serving_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def draw(x, u, T=None, k=None, p=None, m=None, **kw):
    from paper_2602_07306_amd import binding as PB
    dev = lambda a, ty: None if a is None else torch.tensor(np.asarray(a), dtype=ty, device="cuda")
    x = torch.as_tensor(np.asarray(x, dtype=np.float32)).cuda() if not torch.is_tensor(x) else x
    out = PB.pt_sample(x, dev(u, torch.float32), dev(T, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32), **kw)
    torch.cuda.synchronize()
    return out.cpu().numpy()


def check(x, u, T=None, k=None, p=None, m=None):
    x = np.asarray(x, dtype=np.float32)
    got = draw(x, u, T, k, p, m)
    f = lambda a, off, i: off if a is None else float(np.float32(a[i]))
    want = [R.sample(x[i], f(u, 0, i), f(T, 1.0, i), int(f(k, 0, i)), f(p, 1.0, i), f(m, 0.0, i)) for i in range(len(x))]
    assert got.tolist() == want


def logits(rng, rows, vocab, std=2.2):
    x = std * rng.standard_normal((rows, vocab))
    for r in range(rows):
        best = rng.integers(0, vocab, max(1, min(24, vocab // 8)))
        x[r, best] = rng.uniform(5, 11, len(best))
    return x.astype(np.float32)


@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 64, 257, 1000, 1024, 1025, 4099, 32000, 50001, 130001])
@pytest.mark.parametrize("mode", ["none", "k", "p", "m", "all"])
def test_filters(vocab, mode):
    rng = np.random.default_rng(vocab)
    rows = 24
    x = logits(rng, rows, vocab)
    u, T = rng.random(rows), rng.uniform(0.5, 1.5, rows)
    u[:2] = 0.0, np.float32(1) - np.float32(2.0 ** -24)
    k = rng.choice([0, 1, 2, 20, 50, 192, 193, 400, 640, 641, 900, 3000, vocab, 2 ** 31 - 1, -3], rows) if mode in ("k", "all") else None
    p = rng.choice([0.0, 1e-6, 0.1, 0.5, 0.9, 0.95, 0.999, 1.0, 2.0, -1.0], rows) if mode in ("p", "all") else None
    m = rng.choice([0.0, 1e-9, 0.01, 0.1, 0.7, 1.0, 5.0], rows) if mode in ("m", "all") else None
    if m is not None:
        m = np.minimum(m, 1.0)       # above 1: the largest stays, see below
    check(x, u, T, k, p, m)


def test_flat_and_sharp_rows():
    """A nucleus of ten thousands of tokens, and one of a single token."""
    rng = np.random.default_rng(1)
    for std, T in ((0.01, 1.0), (1.0, 30.0), (2.0, 0.02), (50.0, 1.0), (1e30, 1.0), (1e-30, 1.0)):
        x = (std * rng.standard_normal((6, 40000))).astype(np.float32)
        check(x, rng.random(6), [T] * 6, [0, 0, 5000, 20000, 100, 0], [0.5, 0.99, 0.9, 1.0, 0.3, 1e-4])


@pytest.mark.parametrize("vocab", [7, 3000, 32768, 70001])
def test_ties_go_to_the_lowest_index(vocab):
    rng = np.random.default_rng(2)
    same = np.zeros((6, vocab), np.float32)
    same[1] = -3.5
    two = rng.integers(0, 2, (6, vocab)).astype(np.float32)
    few = rng.integers(-4, 5, (6, vocab)).astype(np.float32)
    few[few == 0] = -0.0
    few[:, ::3] = np.where(few[:, ::3] == 0, 0.0, few[:, ::3])
    u = np.array([0, 0.3, 0.5, 0.75, 0.9, 0.99999])
    for x in (same, two, few):
        check(x, u)
        check(x, u, k=[1, 3, 200, vocab // 2, vocab - 1, 650])
        check(x, u, p=[0.25, 0.5, 0.125, 0.75, 0.0, 0.5])       # powers of two: equal in every order of summing
        check(x, u, [1.0] * 6, [vocab // 2, 4, 512, 800, 7, 1], [0.5, 0.5, 0.25, 0.5, 1.0, 0.1], [0.0, 1.0, 0.5, 0.0, 0.2, 0.0])


def test_masked_tokens():
    rng = np.random.default_rng(3)
    x = logits(rng, 9, 5000)
    x[0] = -INF
    x[1, 1:] = -INF
    x[2, ::2] = -INF
    x[3] = NAN
    x[4, 100:] = NAN
    x[5, [7, 99, 4000]] = INF
    x[6] = np.finfo(np.float32).min
    x[7, 3:] = np.finfo(np.float32).min
    x[8, 10:] = -INF
    u = rng.random(9)
    for k, p, m in ((None, None, None), ([50] * 9, None, None), (None, [0.9] * 9, None), ([2] * 9, [0.9] * 9, [0.1] * 9), ([3000] * 9, None, None), (None, None, [0.01] * 9)):
        check(x, u, None, k, p, m)


def test_greedy_rows_equal_argmax():
    from paper_2602_07306_amd import binding as PB
    rng = np.random.default_rng(4)
    x = np.round(logits(rng, 64, 32000))
    got = draw(x, rng.random(64), [0.0] * 32 + [-1.0] * 16 + [NAN] * 16, [5] * 64, [0.5] * 64)
    assert got.tolist() == np.argmax(x, -1).tolist() == PB.pt_argmax(torch.from_numpy(x).cuda()).cpu().tolist()


def test_uniform_numbers_outside_their_range_and_strict_min_p():
    x = np.zeros((4, 100), np.float32)
    assert draw(x, [-1.0, NAN, 1.0, 7.0]).tolist() == [0, 0, 99, 99]
    x = np.array([[1.0, 3.0, 2.0]] * 2, np.float32)
    assert draw(x, [0.99, 0.0], m=[1.5, 1.0]).tolist() == [1, 1]        # the largest always stays


def test_extreme_temperatures():
    rng = np.random.default_rng(5)
    x = logits(rng, 4, 2000)
    check(x, rng.random(4), [1e-30, 1e-3, 1e30, 1e-40])
    check(x, rng.random(4), [1e-30, 1e-3, 1e30, 1e-40], p=[0.5] * 4)
    # all weights equal: the first i with i + 1 > 2000 u; 0.9995 in fp32 is 0.99949998, so 1998.99996 there
    assert draw(x, [0.0, 0.5, 0.5, 0.9995], [INF] * 4).tolist() == [0, 1000, 1000, 1998]


@pytest.mark.parametrize("vocab", [50, 3000, 40000, 70001])
def test_a_uniform_number_of_zero_takes_the_first_token_with_any_weight(vocab):
    """However light it is: 2^-60 of the largest, or 2^-900, but not what fp64 cannot hold."""
    x = np.full((8, vocab), -2000.0, np.float32)
    x[:, vocab // 2] = 10.0
    for r, (i, v) in enumerate(((7, -30.0), (3, -600.0), (9, -800.0), (0, 9.0))):
        x[r, i] = x[r + 4, i] = v
    k, p, m = [0, 5, 3, 2] * 2, [1.0] * 8, [0.0] * 8
    check(x, [0.0] * 8)
    check(x, [0.0] * 8, k=k)
    check(x, [0.0] * 8, k=[700] * 8)
    check(x, [0.0] * 8, p=[0.999] * 4 + [0.3] * 4)
    check(x, [0.0] * 8, k=k, p=[0.999] * 4 + [0.3] * 4, m=[0.0, 0.0, 1e-6, 0.1] * 2)
    check(x, [0.0] * 8, m=[1e-25] * 4 + [0.2] * 4)


def test_rows_apart_and_unaligned():
    rng = np.random.default_rng(6)
    for off in (0, 1, 2, 3):
        wide = torch.zeros((5, 4013), device="cuda")
        x = logits(rng, 5, 4000)
        wide[:, off:off + 4000] = torch.from_numpy(x)
        wide[:, off + 4000:] = 100.0                  # behind the row: not to be read
        if off:
            wide[:, off - 1] = 100.0
        u, k = rng.random(5).astype(np.float32), [0, 40, 1000, 0, 7]
        got = draw(wide[:, off:off + 4000], u, None, k, [0.9, 0.9, 0.9, 1.0, 1.0])
        want = [R.sample(x[i], u[i], 1.0, k[i], float(np.float32([0.9, 0.9, 0.9, 1.0, 1.0][i]))) for i in range(5)]
        assert got.tolist() == want


def test_frequencies_follow_the_weights():
    """Evenly spread uniform numbers give each token its share, to a token's share of one."""
    rng = np.random.default_rng(7)
    x = np.repeat(logits(rng, 1, 50), 4000, axis=0)
    got = draw(x, (np.arange(4000) + 0.5) / 4000)
    w = np.exp(x[0].astype(float) - x[0].max())
    assert np.max(np.abs(np.bincount(got, minlength=50) / 4000 - w / w.sum())) <= 1.0 / 4000


def test_the_same_from_call_to_call_and_in_a_graph():
    from paper_2602_07306_amd import binding as PB
    rng = np.random.default_rng(8)
    x = torch.from_numpy(logits(rng, 40, 32001)).cuda()
    u = torch.rand(40, device="cuda")
    k = torch.from_numpy(rng.choice([0, 10, 300, 2000], 40).astype(np.int32)).cuda()
    p = torch.from_numpy(rng.choice([1.0, 0.9], 40).astype(np.float32)).cuda()
    out = torch.empty(40, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(PB.pt_sample_bytes(40, 32001), 16), dtype=torch.uint8, device="cuda")
    call = lambda: PB.pt_sample(x, u, None, k, p, None, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        u.uniform_()
        x.normal_(0, 3)
        g.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy().copy()
        call()
        torch.cuda.synchronize()
        assert got.tolist() == out.cpu().tolist()
        xs, us, ks, ps = x.cpu().numpy(), u.cpu().numpy(), k.cpu().numpy(), p.cpu().numpy()
        assert got.tolist() == [R.sample(xs[i], us[i], 1.0, ks[i], float(ps[i])) for i in range(40)]
