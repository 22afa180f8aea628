"""pt_sample of few rows and many logits, whose rows are cut into parts: the same tokens as of the same rows in a batch that
is large enough to leave them whole, and those of the definition."""
import numpy as np
import pytest

from tests import serving_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

VOCAB = 70001          # four parts of 18432, 18432, 18432 and 14705
BELOW_ONE = float(np.float32(1) - np.float32(2.0 ** -24))


def tokens(x, u, rows, **filters):
    """The one row x at every number of u, in calls of `rows` rows."""
    from paper_2602_07306_amd import binding as PB
    n = (len(u) + rows - 1) // rows * rows
    us = torch.tensor(np.resize(np.asarray(u, dtype=np.float32), n), device="cuda")
    xs = torch.as_tensor(x, dtype=torch.float32).cuda().expand(rows, -1).contiguous()
    param = {k: torch.full((rows,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in filters.items()}
    out = [PB.pt_sample(xs, us[i:i + rows], **param) for i in range(0, n, rows)]
    return torch.cat(out).cpu().numpy()[:len(u)].tolist()


def masked_tail():
    x = np.zeros(VOCAB, np.float32)
    x[52000:] = -1e9                       # finite, and without any weight
    return x


def masked_tail_with_a_few_tokens():
    x = masked_tail()
    x[[60000, 60001, 69990]] = 0.5
    return x


def light_parts():
    """Weights of 2^-86, 1 and 2^-40 of the largest in parts of their own."""
    x = np.full(VOCAB, -60.0, np.float32)
    x[20000:40000] = 0.0
    x[60000:] = -40 * np.log(2.0)
    return x


def ordinary():
    return (2.2 * np.random.default_rng(3).standard_normal(VOCAB)).astype(np.float32)


@pytest.mark.parametrize("u,last", [(1.0, 51999), (7.0, 51999), (BELOW_ONE, 51999)])
def test_numbers_from_one_on_take_the_last_token_with_a_weight(u, last):
    for rows in (1, 64, 200):
        assert tokens(masked_tail(), [u], rows) == [last]
        assert tokens(masked_tail_with_a_few_tokens(), [u], rows) == [69990]


@pytest.mark.parametrize("row", [masked_tail, masked_tail_with_a_few_tokens, light_parts, ordinary])
def test_a_token_does_not_depend_on_the_number_of_rows(row):
    x = row()
    u = [0.0, 1e-38, 1e-30, 1e-20, 1e-12, 1e-7, 0.25, 0.5, 0.75, 0.999, BELOW_ONE, 1.0, 7.0] + np.random.default_rng(4).random(187).tolist()
    whole = tokens(x, u, 200)
    for rows in (1, 16, 64, 128):
        assert tokens(x, u, rows) == whole
    for temperature in (0.3, 30.0):
        assert tokens(x, u, 64, temperature=temperature) == tokens(x, u, 200, temperature=temperature)


@pytest.mark.parametrize("vocab,rows", [(32768, 1), (130001, 64), (130001, 3), (300007, 2)])
def test_rows_in_parts_against_the_definition(vocab, rows):
    from paper_2602_07306_amd import binding as PB
    rng = np.random.default_rng(vocab + rows)
    x = (2.2 * rng.standard_normal((rows, vocab))).astype(np.float32)
    for r in range(rows):
        best = rng.choice(vocab, 24, replace=False)
        x[r, best] = rng.uniform(5, 11, 24)
    u, T = rng.random(rows).astype(np.float32), rng.uniform(0.6, 1.3, rows).astype(np.float32)
    got = PB.pt_sample(torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda(), torch.from_numpy(T).cuda()).cpu().tolist()
    assert got == [R.sample(x[i], u[i], float(T[i])) for i in range(rows)]


def test_infinite_and_missing_logits_in_some_parts():
    x = ordinary()
    x[:20000] = -np.inf
    x[40000:50000] = np.nan
    u = [0.0, 1e-7, 0.3, 0.9, 1.0] + np.random.default_rng(5).random(59).tolist()
    assert tokens(x, u, 64) == tokens(x, u, 256)
    x[[100, 30000, 69999]] = np.inf
    got = tokens(x, [0.0, 0.4, 0.9, 1.0], 4)
    assert got == tokens(x, [0.0, 0.4, 0.9, 1.0], 256) == [100, 30000, 69999, 69999]
    assert tokens(np.full(VOCAB, -np.inf, np.float32), [0.5], 1) == [-1]


def test_captured_with_filters_that_change():
    """Rows with and without filters in one captured call, whose parameters change between the replays."""
    from paper_2602_07306_amd import binding as PB
    rows, rng = 20, np.random.default_rng(6)
    x = torch.from_numpy((2.2 * rng.standard_normal((rows, VOCAB))).astype(np.float32)).cuda()
    u, k, out = torch.rand(rows, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    ws = torch.empty(PB.pt_sample_bytes(rows, VOCAB), dtype=torch.uint8, device="cuda")
    call = lambda: PB.pt_sample(x, u, None, k, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        u.uniform_()
        x.normal_(0, 2)
        k.copy_(torch.from_numpy(rng.choice([0, 0, 30, 500], rows).astype(np.int32)))
        ws.fill_(0x5a)
        g.replay()
        torch.cuda.synchronize()
        xs, us, ks = x.cpu().numpy(), u.cpu().numpy(), k.cpu().numpy()
        assert out.cpu().tolist() == [R.sample(xs[j], us[j], 1.0, int(ks[j])) for j in range(rows)]
