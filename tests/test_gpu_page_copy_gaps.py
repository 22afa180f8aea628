"""pt_page_copy between the stretches that it copies: what lies there stays as it was, in pools whose pages have gaps."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# dimensions of the buffer: layer, page, head, slot, and the head's width with a gap of 8 behind it
LAYOUTS = {"by_page": "PLHSD", "by_token": "LPSHD", "page_inside": "LSPHD"}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1, 9, 1, 16, 8), (3, 12, 2, 16, 72), (2, 40, 4, 64, 128)])
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_what_lies_between_is_left_alone(dtype, shape, layout):
    from paper_2602_07306_amd import binding as PB
    size = dict(zip("LPHSD", shape))
    size["D"] += 8
    dims = LAYOUTS[layout]
    as_cache = lambda w: w.permute([dims.index(d) for d in "LPHSD"])
    gen = torch.Generator(device="cuda").manual_seed(size["P"])
    whole = [torch.randn([size[d] for d in dims], generator=gen, device="cuda").to(dtype) for _ in range(2)]
    before = [w.clone() for w in whole]
    P, D = shape[1], shape[4]
    order = np.random.default_rng(P).permutation(P)
    n = P // 2
    pairs = np.stack([order[:n], order[n:2 * n]], axis=1).astype(np.int32)
    PB.pt_page_copy(PB.PTPagedCache(*(as_cache(w)[..., :D] for w in whole)), pairs)
    torch.cuda.synchronize()
    src, dst = (torch.from_numpy(pairs[:, i].astype(np.int64)).cuda() for i in range(2))
    for b, w in zip(before, whole):
        expected = b.clone()
        as_cache(expected)[:, dst, :, :, :D] = as_cache(b)[:, src, :, :, :D]
        assert torch.equal(w, expected)          # the gap behind each head's width among it
