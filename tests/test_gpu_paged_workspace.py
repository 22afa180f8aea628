"""Workspaces of pt_paged_attention: partials of few and of many rows lie apart, inside the bytes that were asked for, and need
nothing of what the memory held before."""
import pytest

from tests.test_gpu_paged_attention import Problem

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BESIDE = [(1, 5003), (300, 700), (2, 2500), (1, 40), (0, 10), (150, 2100), (1, 1)]


@pytest.mark.parametrize("H,Hkv,hd,dtype,lens", [
    (4, 4, 64, "bf16", BESIDE), (8, 2, 128, "bf16", BESIDE), (8, 1, 96, "bf16", BESIDE), (20, 1, 64, "bf16", BESIDE),
    (40, 1, 64, "bf16", BESIDE),                                     # no class of few rows
    (4, 1, 64, "bf16", [(200, 6000)]), (8, 2, 64, "bf16", [(1, 9000), (1, 17), (3, 3000)]),
    (4, 1, 256, "bf16", [(1, 3000), (60, 2500)]), (4, 2, 64, "fp32", [(1, 3000), (60, 2500)])])
def test_partials_lie_inside_their_workspace(H, Hkv, hd, dtype, lens):
    p = Problem(H, Hkv, hd, dtype, 16, lens, seed=H + hd)
    n = p.PB.pt_paged_attention_bytes(p.cache, p.batch, H)
    assert n > 0
    whole = torch.empty(n + 512, dtype=torch.uint8, device="cuda")
    outs = []
    for fill in (0xff, 0x00, 0x7f):                                  # no numbers, zeros, large numbers
        whole.fill_(fill)
        outs.append(p.run(workspace=whole[256:256 + n]))
        assert torch.all(whole[:256] == fill) and torch.all(whole[256 + n:] == fill)
    p.check(outs[0])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert int(p.status) == 0


def test_a_captured_batch_whose_rows_change_class():
    """The sequences' rows change between replays, from one to many and back, inside the bounds that the call was given."""
    p = Problem(4, 2, 64, "bf16", 16, [(1, 2100), (200, 2200), (1, 1500)], seed=3)
    n = p.PB.pt_paged_attention_bytes(p.cache, p.batch, 4)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(p.q, memory_format=torch.contiguous_format)
    call = lambda: p.PB.pt_paged_attention(p.cache, p.layer, p.batch, p.q, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rows in ((200, 1, 1), (4, 4, 194), (66, 66, 66), (0, 200, 2), (1, 200, 1)):
        start = [0, rows[0], rows[0] + rows[1], sum(rows)]
        p.row_start[:] = start
        p.batch.row_start.copy_(torch.from_numpy(p.row_start))
        out.fill_(7.0)
        ws.fill_(0xff)
        g.replay()
        torch.cuda.synchronize()
        p.check(out)
    assert int(p.status) == 0
