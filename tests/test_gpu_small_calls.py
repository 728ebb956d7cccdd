"""Which of the two kernels a windowed or 4-bit call runs (one that knows its segments from the launch, or the one with a work list), read off
the grid of the captured launch, and that both are right on either side of the limit."""
import pytest
import torch

from paper_2606_29986_b200 import hma
from records import Paged

BFP8, BF16, BFP4 = hma.HMA_KV_BFP8, hma.HMA_KV_BF16, hma.HMA_KV_BFP4


def grid_of(call):
    """CTAs of the one kernel that `call` launches."""
    driver = pytest.importorskip("cuda.bindings.driver")
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call()
    graph = driver.CUgraph(g.raw_cuda_graph())
    err, nodes, n = driver.cuGraphGetNodes(graph, 16)
    assert int(err) == 0 and n == 1
    err, params = driver.cuGraphKernelNodeGetParams(nodes[0])
    assert int(err) == 0
    return params.gridDimX


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,lens,window,cols,small", [
    (BFP4, [1024] * 4, None, 64, True), (BFP4, [1024] * 4, None, 128, True), (BFP4, [1024] * 4, None, 145, False), (BFP4, [1024] * 4, None, 2048, False),
    (BFP4, [500] * 30, None, 32, True), (BFP4, [500] * 30, None, 512, False), (BFP4, [90] * 150, None, 6, True), (BFP4, [90] * 300, None, 6, False),
    (BFP8, [3000] * 4, 900, 200, True), (BFP8, [3000] * 4, 1300, 200, False), (BFP8, [3000] * 4, 900, 4096, True), (BFP8, [100] * 4, 4000, 7, True),
    (BF16, [3000] * 4, 600, 200, True), (BF16, [3000] * 4, 1300, 200, False), (BFP8, [64] * 4, None, 4, False), (BF16, [64] * 4, None, 4, False)])
def test_either_side_of_the_limit(fmt, lens, window, cols, small):
    hkv = 8
    p = Paged(lens, hkv, hkv, fmt, seed=cols, window=window, extra_cols=cols - (max(lens) + 15) // 16)
    assert p.tbl.shape[1] == cols
    ws, out = hma.new_workspace(p.desc, len(lens)), torch.full(p.q.shape, 3.0, device="cuda")

    def call(out=out):
        if window:
            hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, window, 0, p.scale, ws)
        else:
            hma.hma_decode_attention_multi(p.cache, 0, p.q, out, p.tbl, p.ctx, p.scale, ws)
    call()                                           # (attributes are set by the first call, outside a capture)
    torch.cuda.synchronize()
    sms, segments = torch.cuda.get_device_properties(0).multi_processor_count, len(lens) * hkv
    per = 1
    while -(-segments // per) > sms:                 # segments a CTA: the fewest that make one wave
        per *= 2
    assert grid_of(call) == (-(-segments // per) if small else sms)
    out16 = torch.empty(p.q.shape, dtype=torch.bfloat16, device="cuda")
    call(out16)
    torch.cuda.synchronize()
    p.check(out, out16, *p.reference(window=window))
