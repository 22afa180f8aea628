"""Calls of the serving operators at the ends of what their documentation allows."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_step_without_rows():
    """A server's step in which nothing is left to do: empty tensors through append, attention and sampling."""
    from paper_2602_07306_amd import binding as PB
    k5, v5 = (torch.full((1, 4, 2, 16, 64), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = PB.PTPagedCache(k5, v5)
    rows = lambda heads: torch.empty((0, heads, 64), dtype=torch.bfloat16, device="cuda")
    none = PB.PTPagedBatch(i32([0]), i32([]), torch.empty((0, 3), dtype=torch.int32, device="cuda"), total_rows=0)
    idle = PB.PTPagedBatch(i32([0, 0, 0]), i32([5, 0]), i32([[1], [2]]), total_rows=0)     # sequences, and no new row of any
    for batch in (none, idle):
        q = PB.pt_paged_append(cache, 0, batch, rows(2), rows(2), q=rows(4), rope=PB.PTRope(PB.PT_ROPE_HALF, 64))
        assert q.shape == (0, 4, 64)
        assert PB.pt_paged_attention(cache, 0, batch, q).shape == (0, 4, 64)
        by_head = torch.empty((4, 0, 192), dtype=torch.bfloat16, device="cuda").transpose(0, 1)[..., :64]
        assert PB.pt_paged_attention(cache, 0, batch, by_head, out=rows(4)).shape == (0, 4, 64)
    assert PB.pt_sample(torch.empty((0, 100), device="cuda"), torch.empty(0, device="cuda")).shape == (0,)
    torch.cuda.synchronize()
    assert torch.all(k5 == 3.0) and torch.all(v5 == 3.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hkv,hd,lens", [(4, 2, 64, [(1, 200), (9, 40)]), (8, 1, 128, [(60, 300), (1, 700)]), (4, 2, 64, [(3, 3000), (1, 17)])])
@pytest.mark.parametrize("factor", [30.0, 300.0])
def test_large_scores_follow_the_definition(dtype, H, Hkv, hd, lens, factor):
    """Scores of several hundred and thousand: the running maximum moves far, in one range and over several.  The bound of a
    result grows with the scores, by (hd + 6) 2^-24 of their terms' sum: a few per cent of the weights here."""
    from tests.test_gpu_paged_attention import Problem
    p = Problem(H, Hkv, hd, dtype, 16, lens, seed=6, scale_q=factor)
    out = p.run()
    used = int(p.row_start[-1])
    assert torch.isfinite(out[:used].float()).all()
    p.check(out)
