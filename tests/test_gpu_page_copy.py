"""pt_page_copy: exact copies in every layer and layout, everything else untouched."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1, 9, 1, 16, 8), (3, 12, 2, 16, 72), (2, 40, 4, 64, 128), (5, 1000, 1, 16, 64)])
@pytest.mark.parametrize("order", ["head", "token", "gaps", "mixed"])
def test_copies(dtype, shape, order):
    from paper_2602_07306_amd import binding as PB
    L, P, H, S, D = shape
    gen = torch.Generator(device="cuda").manual_seed(P)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    if order == "head":
        k, v = new(*shape), new(*shape)
    elif order == "token":
        k, v = (new(L, P, S, H, D).transpose(2, 3) for _ in range(2))
    elif order == "gaps":       # K and V side by side in one buffer
        both = new(P, L, H, S, 2, D + 8)
        k, v = (both[:, :, :, :, i, :D].transpose(0, 1) for i in range(2))
    else:                       # the page innermost but one
        k, v = (new(L, S, P, H, D).permute(0, 2, 3, 1, 4) for _ in range(2))
    rng = np.random.default_rng(P)
    order_ = rng.permutation(P)
    n = P // 2 if P < 900 else 450
    pairs = np.stack([rng.choice(order_[:P - n], n), order_[P - n:]], axis=1)     # a source may be copied more than once
    want_k, want_v = k.clone(), v.clone()
    src, dst = (torch.from_numpy(pairs[:, i].copy()).cuda() for i in range(2))
    want_k[:, dst], want_v[:, dst] = k[:, src], v[:, src]
    PB.pt_page_copy(PB.PTPagedCache(k, v), pairs.tolist() if P < 100 else pairs)
    torch.cuda.synchronize()
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    if order == "gaps":
        assert torch.equal(both[..., D:], both[..., D:].clone())


def test_a_pool_past_32_bits():
    from paper_2602_07306_amd import binding as PB
    pages = (1 << 31) // (2 * 128 * 128) + 4
    k = torch.empty((1, pages, 2, 128, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    k[0, 0].normal_()
    v[0, 0].normal_()
    k[0, pages - 2].normal_()
    v[0, pages - 2].normal_()
    PB.pt_page_copy(PB.PTPagedCache(k, v), [(0, pages - 1), (pages - 2, 1)])
    torch.cuda.synchronize()
    assert torch.equal(k[0, 0], k[0, pages - 1]) and torch.equal(v[0, 0], v[0, pages - 1])
    assert torch.equal(k[0, pages - 2], k[0, 1]) and torch.equal(v[0, pages - 2], v[0, 1])


def test_captured_graph_keeps_its_pairs():
    from paper_2602_07306_amd import binding as PB
    k, v = (torch.randn((2, 16, 2, 16, 64), device="cuda") for _ in range(2))
    cache, pairs = PB.PTPagedCache(k, v), np.array([[0, 8], [3, 9]], dtype=np.int32)
    PB.pt_page_copy(cache, [(1, 15)])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        PB.pt_page_copy(cache, pairs)
    pairs[:] = 7
    for _ in range(3):
        k.normal_()
        v.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(k[:, 8], k[:, 0]) and torch.equal(v[:, 9], v[:, 3]) and not torch.equal(k[:, 7], k[:, 8])
