"""hma_decode_attention_window: sliding window and first tokens, on every cache format, against 64-bit attention over the visible tokens."""
import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma
from records import Paged

FORMATS = [hma.HMA_KV_BFP8, hma.HMA_KV_BFP4, hma.HMA_KV_BF16]


def run(p, window, sinks, q=None, stream=None, ws=None):
    q = p.q if q is None else q
    ws = hma.new_workspace(p.desc, q.shape[0] * q.shape[1]) if ws is None else ws
    outs = []
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full(q.shape, float("nan"), dtype=dt, device="cuda")
        hma.hma_decode_attention_window(p.cache, 0, q, out, p.tbl, p.ctx, window, sinks, p.scale, ws, stream=stream)
        outs.append(out)
    torch.cuda.synchronize()
    assert int(ws[:1024 * 64 * 4].max()) == 0            # the arrival counters are back at zero
    return outs


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 16), (33, 5), (100, 40), (5, 300), (1000, 0), (2**31 - 1, 2**31 - 1)])
def test_windows_and_sinks(fmt, window, sinks):
    lens = [0, 1, 15, 16, 17, 33, 100, 257, 400]
    p = Paged(lens, 8, 2, fmt, seed=window % 1000 + sinks % 1000, window=window, sinks=sinks, extra_cols=2)
    p.check(*run(p, window, sinks), *p.reference(window=window, sinks=sinks))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_len", [2, 3, 4, 17])
def test_several_query_tokens(fmt, q_len):
    """Every query has a window of its own; queries before the sequence's first token are rows of zeros."""
    p = Paged([0, 1, 2, 16, 40, 203], 10, 2, fmt, seed=q_len, q_len=q_len, window=21, sinks=3)
    p.check(*run(p, 21, 3), *p.reference(window=21, sinks=3))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 1), (8, 8), (21, 3), (64, 8), (64, 64)])
def test_heads_and_long_contexts(fmt, hq, hkv):
    p = Paged([5000, 70, 2000], hq, hkv, fmt, seed=hq, window=1500, sinks=20)
    p.check(*run(p, 1500, 20), *p.reference(window=1500, sinks=20))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_a_window_over_everything_is_plain_attention(fmt):
    p = Paged([1500, 5, 0, 64], 8, 2, fmt, seed=3)
    got, _ = run(p, 1500, 0)
    plain = torch.empty_like(got)
    hma.hma_decode_attention(p.cache, 0, p.q[:, 0].contiguous(), plain.view(4, 8, 128), p.tbl, p.ctx, p.scale, hma.new_workspace(p.desc, 4))
    assert torch.equal(got, plain)                         # the same pages, the same split, the same order


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("b,hkv,window,q_len", [(1, 1, 4000, 1), (9, 2, 300, 1), (37, 4, 100, 1), (74, 4, 60, 2), (100, 8, 9, 2), (148, 1, 700, 1), (149, 1, 150, 1), (30, 64, 1, 1), (296, 8, 1, 1)])
def test_small_calls(fmt, b, hkv, window, q_len):
    """Every number of segments per CTA that the small path knows, with rows from empty to the whole window, and its neighbours beyond it."""
    rng = np.random.default_rng(b)
    lens = rng.integers(0, 2 * window + 20, b)
    lens[rng.random(b) < 0.2] = 0
    p = Paged(lens, hkv * 3, hkv, fmt, seed=b, q_len=q_len, window=window, sinks=17)
    p.check(*run(p, window, 17), *p.reference(window=window, sinks=17))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_len", [1, 2, 3])
def test_large_windows(fmt, q_len):
    """Windows that are cut into many warps' shares: several sequences, some shorter than the window, some empty."""
    p = Paged([5000, 0, 2999, 300, 4100, 1, 2017], 4, 1, fmt, seed=q_len, q_len=q_len, window=3000, sinks=40)
    p.check(*run(p, 3000, 40), *p.reference(window=3000, sinks=40))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_len", [1, 2])
@pytest.mark.parametrize("hkv,window,lens", [(1, 1500, [4000]), (8, 600, [3000, 20, 0, 900]), (3, 1100, [1100, 1101, 5000]), (2, 2000, [2500, 0, 40, 1999])])
def test_few_long_sequences(fmt, q_len, hkv, window, lens):
    """Few sequences, windows of many pages: either side of the limit at which the list takes over."""
    p = Paged(lens, hkv * 2, hkv, fmt, seed=hkv, q_len=q_len, window=window, sinks=9)
    p.check(*run(p, window, 9), *p.reference(window=window, sinks=9))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_random_batches(fmt):
    rng = np.random.default_rng(fmt + 5)
    for i in range(6):
        b, hkv = int(rng.integers(1, 60)), int(rng.choice([1, 2, 4]))
        window, sinks, q_len = int(rng.integers(1, 400)), int(rng.integers(0, 50)), int(rng.integers(1, 4))
        p = Paged(rng.integers(0, 900, b), hkv * int(rng.integers(1, 9)), hkv, fmt, seed=i, q_len=q_len, window=window, sinks=sinks)
        p.check(*run(p, window, sinks), *p.reference(window=window, sinks=sinks))


@pytest.mark.gpu
def test_many_rows():
    """As many rows as a call takes, most of them short."""
    lens = [(i * 37) % 90 for i in range(1024)]
    p = Paged(lens, 2, 1, hma.HMA_KV_BFP8, seed=9, window=30, sinks=2)
    p.check(*run(p, 30, 2), *p.reference(window=30, sinks=2))
    with pytest.raises(hma.HmaError) as e:
        hma.hma_decode_attention_window(p.cache, 0, p.q.expand(-1, 2, -1, -1).contiguous(), p.q, p.tbl, p.ctx, 30, 2, 1.0, hma.new_workspace(p.desc, 1024))
    assert e.value.status == hma.HMA_ERR_UNSUPPORTED_SHAPE


@pytest.mark.gpu
def test_bad_visible_pages_are_skipped_and_flagged():
    p = Paged([100, 100], 4, 1, hma.HMA_KV_BFP8, seed=2, window=40, sinks=4)
    ref, tol = p.reference(window=40, sinks=4)
    p.tbl[0, 0] = -1
    out = torch.zeros(p.q.shape, device="cuda")
    hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, 40, 4, p.scale, hma.new_workspace(p.desc, 2))
    assert hma.hma_error_flags(p.cache) == hma.HMA_FLAG_BAD_PAGE_ATTENTION
    assert (np.abs(out[1].double().cpu().numpy() - ref[1]) <= tol[1]).all() and bool(torch.isfinite(out).all())


@pytest.mark.gpu
def test_window_in_a_graph_on_another_stream():
    """Lengths grow between replays: the window moves on its own."""
    p = Paged([200, 31, 90], 8, 2, hma.HMA_KV_BFP4, seed=4, extra_cols=1)
    ws, out = hma.new_workspace(p.desc, 3), torch.zeros(p.q.shape, device="cuda")
    p.ctx.sub_(9)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, 37, 2, p.scale, ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, 37, 2, p.scale, ws)
    full = p.lens.copy()
    for grow in range(0, 10, 3):
        p.ctx.copy_(torch.from_numpy(full - 9 + grow))
        p.lens = (full - 9 + grow).astype(np.int32)
        g.replay()
        ref, tol = p.reference(window=37, sinks=2)
        assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.gpu
def test_refusals():
    p = Paged([40], 4, 1, hma.HMA_KV_BFP8, window=8, sinks=0)
    ws, n0 = hma.new_workspace(p.desc, 1), hma.hma_launch_count()
    L, out = hma.lib(), torch.zeros(p.q.shape, device="cuda")
    ok = dict(layer=0, q=p.q.data_ptr(), out=out.data_ptr(), dt=1, t=p.tbl.data_ptr(), mp=3, c=p.ctx.data_ptr(), b=1, ql=1, w=8, s=0, ws=ws.data_ptr(), n=ws.numel())
    call = lambda **kw: (lambda a: L.hma_decode_attention_window(p.cache.handle, a["layer"], a["q"], a["out"], a["dt"], a["t"], a["mp"], a["c"], a["b"], a["ql"], a["w"],
                                                                 a["s"], 0.1, a["ws"], a["n"], None))({**ok, **kw})
    assert [call(w=0), call(w=-4), call(s=-1), call(ql=0), call(layer=1), call(q=None), call(out=None), call(t=None), call(ws=None), call(dt=5), call(b=-1)] == [1] * 11
    assert [call(q=ok["q"] + 2), call(out=ok["out"] + 4), call(ws=ok["ws"] + 16)] == [3] * 3 and call(n=1000) == hma.HMA_ERR_WORKSPACE_TOO_SMALL
    assert call(ql=1025) == hma.HMA_ERR_UNSUPPORTED_SHAPE and call(b=0, q=None) == 0 and hma.hma_launch_count() == n0


def test_refusals_without_a_gpu():
    L = hma.lib()
    assert L.hma_decode_attention_window(None, 0, None, None, 0, None, 0, None, 1, 1, 4, 0, 1.0, None, 0, None) == hma.HMA_ERR_INVALID_ARG


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    p = Paged([40, 3], 8, 2, 0, seed=1)
    q, out, ws = p.q[:, 0].contiguous(), torch.empty(2, 8, 128, device="cuda"), hma.new_workspace(p.desc, 2)
    ok = dict(q=q, out=out, tbl=p.tbl, ctx=p.ctx)
    wide = torch.zeros(2, 8, 256, dtype=torch.bfloat16, device="cuda")
    call = lambda q, out, tbl, ctx: hma.hma_decode_attention_window(p.cache, 0, q, out, tbl, ctx, 5, 0, p.scale, ws)
    call(**ok)
    for bad in (dict(q=q.float()), dict(q=wide[:, :, :128]), dict(q=q[:, :4].contiguous()), dict(q=q.view(-1)), dict(q=q.cpu()), dict(out=out[:1]), dict(out=out.half()),
                dict(out=out.transpose(0, 1)), dict(tbl=p.tbl[:1]), dict(tbl=p.tbl.long()), dict(tbl=p.tbl.t()), dict(ctx=p.ctx[:1]), dict(ctx=p.ctx.long()), dict(ctx=p.ctx.cpu())):
        with pytest.raises(hma.HmaError):
            call(**{**ok, **bad})


@pytest.mark.gpu
@pytest.mark.parametrize("far", [2**31, 2**32 + 1, 2**32 + 2**31, 2**40 + 3, 2**63 - 1, 2**70])
def test_numbers_beyond_32_bits(far):
    """A window or a count of first tokens without an end is every token; the same number below zero is refused."""
    p = Paged([300, 5, 40], 4, 2, hma.HMA_KV_BFP8, seed=5)
    ref, tol = p.reference()
    for window, sinks in ((far, 0), (1, far), (far, far)):
        p.check(*run(p, window, sinks), ref, tol)
    ws, out = hma.new_workspace(p.desc, 3), torch.empty(p.q.shape, device="cuda")
    for window, sinks in ((-far, 0), (5, -far)):
        with pytest.raises(hma.HmaError) as e:
            hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, window, sinks, p.scale, ws)
        assert e.value.status == hma.HMA_ERR_INVALID_ARG


def test_int32_keeps_the_sign_and_the_size():
    assert [hma._int32(n) for n in (0, 5, -1, 2**31 - 1, 2**31, 2**40 + 3, -2**31, -2**31 - 1, -2**40)] == [0, 5, -1] + [2**31 - 1] * 3 + [-2**31] * 3
