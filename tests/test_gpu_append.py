"""hma_kv_append and hma_qk_norm_rope: cache bytes against the record formulas, rows against the formulas in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma
import records

FORMATS = [hma.HMA_KV_BFP8, hma.HMA_KV_BFP4, hma.HMA_KV_BF16]
rng0 = np.random.default_rng


def test_records_agree_with_the_wire_oracle():
    """The helper's encoder is the wire encoder of the C oracle, its decode the oracle's, on values of every size."""
    from oracle import oracle as orc
    from paper_2606_29986_b200 import synth
    rng = rng0(1)
    x = (rng.standard_normal((200, 128)) * 2.0 ** rng.integers(-140, 120, (200, 128))).astype(np.float32)
    x[:50] = (rng.standard_normal((50, 128))).astype(np.float32)
    x[3, ::2] = 0.0
    wire = synth.bfp8_encode(torch.from_numpy(x)).numpy()
    for row, w in zip(x, wire):
        E, code = records.encode(row, hma.HMA_KV_BFP8)
        assert np.array_equal(np.concatenate([E, code]), w)
    for fmt in FORMATS:
        for what in (0, 1):
            at, nib = records.places(fmt, what)
            key = at * 2 + (0 if nib is None else nib)
            assert len(np.unique(key)) == 2048 and at.min() >= what * records.HALF[fmt] and at.max() < (1 + what) * records.HALF[fmt]
            assert len(np.unique(records.exp_places(fmt, what))) == 128
            if nib is not None:        # the two codes of a byte belong to one token
                for t in range(16):
                    assert all((at[t] == b).sum() == 2 for b in np.unique(at[t]))


def test_four_bit_encoding_by_hand():
    x = np.zeros(128, np.float32)
    x[:8] = [1.0, -1.0, 1.75, 1.99, -0.125, 0.124, 0.375, 0.625]
    E, code = records.encode(x, hma.HMA_KV_BFP4)
    # the block's exponent is 127, a step is 2^-2: 4, -4, 7, 7 (saturated), -0.5 -> 0, 0, 1.5 -> 2, 2.5 -> 2
    assert E[0] == 127 and E[1] == 0 and (code - 8.0)[:8].tolist() == [4, -4, 7, 7, 0, 0, 2, 2] and (code[16:] == 8).all()


def make_cache(fmt, hkv, pages, hq=None, key_layout=0, layers=1, seed=0):
    desc = hma.make_desc(layers, hq or hkv, hkv, pages, fmt, key_layout=key_layout)
    rng = rng0(seed + 77)
    raw = [rng.integers(0, 256, hma.hma_cache_layer_bytes(desc), dtype=np.uint8) for _ in range(layers)]
    guard = 256
    bufs = [torch.from_numpy(np.concatenate([r, np.full(guard, 0x3C, np.uint8)])).cuda() for r in raw]
    cache = hma.KVCache(desc, layers=[b[:-guard] for b in bufs])
    return cache, raw, bufs


SLOTS = {
    "one": lambda n, P, r: [P * 16 - 1],
    "scattered": lambda n, P, r: r.permutation(P * 16)[:n],
    "prompt": lambda n, P, r: [int(p) * 16 + i % 16 for p, i in zip(np.repeat(r.permutation(P), 16)[:n], range(n))],
    "late start": lambda n, P, r: [int(p) * 16 + i % 16 for p, i in zip(np.repeat(r.permutation(P), 16)[5:5 + n], range(5, 5 + n))],
    "in order": lambda n, P, r: range(3, 3 + n),
    "backwards": lambda n, P, r: range(n)[::-1],
    "padded": lambda n, P, r: [int(s) if i % 3 else -1 for i, s in enumerate(r.permutation(P * 16)[:n])],
    "padded pages": lambda n, P, r: [-1] * 7 + list(range(16, 16 + n - 20)) + [-1] * 13,
    "bad": lambda n, P, r: [int(s) if i % 4 else [-2, P * 16, 2**40, -2**40][i // 4 % 4] for i, s in enumerate(r.permutation(P * 16)[:n])],
    "beyond the end": lambda n, P, r: range(P * 16 - 8, P * 16 - 8 + n),
    "runs": lambda n, P, r: np.concatenate([np.arange(16) + 16 * p if i % 2 else np.arange(9) + 16 * p for i, p in enumerate(r.permutation(P))])[:n],
}


def rows(n, hkv, dtype, seed, odd_values=False):
    rng = rng0(seed)
    x = rng.standard_normal((n, hkv, 128)).astype(np.float32)
    x[:, :, ::31] *= 20
    if odd_values:
        x *= 2.0 ** rng.integers(-135, 125, x.shape).astype(np.float64)
        x = x.astype(np.float32)
        x[rng.random(x.shape) < 0.02] = 0.0
        x[rng.random(x.shape) < 0.02] = -0.0
        x[0, 0, :3] = [np.nan, np.inf, -np.inf]
    t = torch.from_numpy(x).to(dtype)
    return t, t.float().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", list(SLOTS))
def test_append_writes_these_bytes_and_no_others(fmt, kind):
    for n, hkv, dtype, layout in ((1, 1, torch.bfloat16, 0), (40, 2, torch.float32, 0), (67, 3, torch.bfloat16, 1), (160, 1, torch.float32, 1)):
        P = 12
        slots = np.array(list(SLOTS[kind](n, P, rng0(n))), np.int64)[:n]
        n = len(slots)
        cache, raw, bufs = make_cache(fmt, hkv, P, key_layout=layout, layers=2)
        k, kf = rows(n, hkv, dtype, 2 * n)
        v, vf = rows(n, hkv, dtype, 2 * n + 1)
        flags = records.write(raw[1], cache.desc, slots, kf, vf)
        hma.hma_kv_append(cache, 1, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda())
        torch.cuda.synchronize()
        for b, r in zip(bufs, raw):
            assert np.array_equal(b[:-256].cpu().numpy(), r), (n, hkv)
            assert bool((b[-256:] == 0x3C).all())
        assert hma.hma_error_flags(cache) == flags


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_odd_values(fmt):
    """Subnormals, zeros of both signs, NaN and Inf, blocks over the whole exponent range."""
    for dtype in (torch.float32, torch.bfloat16):
        cache, raw, bufs = make_cache(fmt, 2, 9)
        k, kf = rows(130, 2, dtype, 5, True)
        v, vf = rows(130, 2, dtype, 6, True)
        slots = np.concatenate([np.arange(16, 16 + 64), rng0(1).permutation(np.arange(80, 144))[:66 - 2], [0, 5]]).astype(np.int64)
        flags = records.write(raw[0], cache.desc, slots, kf, vf)
        hma.hma_kv_append(cache, 0, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda())
        got, want = bufs[0][:-256].cpu().numpy(), raw[0]
        if fmt == hma.HMA_KV_BF16:       # a NaN is a NaN, whichever
            g, w = got.view(np.uint16), want.view(np.uint16)
            nan = (w & 0x7FFF) > 0x7F80
            written = np.array_equal(g[~nan], w[~nan]) and ((g[nan] & 0x7FFF) > 0x7F80).all()
            assert written
        else:
            assert np.array_equal(got, want)
        assert hma.hma_error_flags(cache) == flags


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [hma.HMA_KV_BFP8])
def test_append_is_encode_and_ingest(fmt):
    """The same bytes as the two calls that did it before."""
    n, hkv = 53, 4
    a, b = (hma.KVCache(hma.make_desc(1, hkv, hkv, 8), fill=0) for _ in range(2))
    k, _ = rows(n, hkv, torch.float32, 3)
    v, _ = rows(n, hkv, torch.float32, 4)
    pages = torch.tensor([5, 0, 7, 2], dtype=torch.int32, device="cuda")
    slots = (pages.long().repeat_interleave(16) * 16 + torch.arange(16, device="cuda").repeat(4))[:n].contiguous()
    hma.hma_kv_append(a, 0, k.cuda(), v.cuda(), slots)
    wires = []
    for x in (k, v):
        x = x.transpose(0, 1).contiguous().cuda()
        w = torch.empty((hkv, n, 136), dtype=torch.uint8, device="cuda")
        hma.hma_bfp8_encode_rows(b, x, w)
        wires.append(w)
    hma.hma_kv_ingest_layer(b, 0, *wires, hma.HMA_WIRE_ROWMAJOR, 0, hkv, pages, 0, n)
    assert torch.equal(a.layers[0], b.layers[0])


@pytest.mark.gpu
def test_append_from_slices_in_a_graph_on_another_stream():
    n, hq, hkv, P = 21, 6, 2, 4
    cache, raw, bufs = make_cache(hma.HMA_KV_BFP4, hkv, P)
    qkv = torch.zeros((n, 16 + (hq + 2 * hkv) * 128), dtype=torch.bfloat16, device="cuda")        # rows with a gap between them
    k = qkv[:, hq * 128:(hq + hkv) * 128].unflatten(1, (hkv, 128))
    v = qkv[:, (hq + hkv) * 128:(hq + 2 * hkv) * 128].unflatten(1, (hkv, 128))
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        hma.hma_kv_append(cache, 0, k, v, slots)
    for seed in (1, 2):
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(seed)).bfloat16())
        at = rng0(seed).permutation(P * 16)[:n]
        slots.copy_(torch.from_numpy(at))
        g.replay()
        torch.cuda.synchronize()
        records.write(raw[0], cache.desc, at, k.float().cpu().numpy(), v.float().cpu().numpy())
        assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0])


# ---------------------------------------------------------------- norm and rotation
def norm_rope_oracle(x, w, eps, table, pos, inter):
    """float64 [n][heads][128] of one kind of head, and the scale that rounding errors go by."""
    y = x.astype(np.float64)
    if w is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * w.astype(np.float64)
    size = np.abs(y)
    if table is not None:
        r = table.shape[1]
        c, s = table[pos, :r // 2].astype(np.float64)[:, None], table[pos, r // 2:].astype(np.float64)[:, None]
        a, b = (np.s_[..., 0:r:2], np.s_[..., 1:r:2]) if inter else (np.s_[..., :r // 2], np.s_[..., r // 2:r])
        out, both = y.copy(), size.copy()
        out[a], out[b] = y[a] * c - y[b] * s, y[b] * c + y[a] * s
        both[a] = both[b] = size[a] + size[b]
        y, size = out, both
    return y, size


def assert_rows(got, want, size):
    # rounded once to BF16 (2^-8 of the value) from fp32: the sum of squares (<= 12 additions deep), its root and the two
    # products leave at most 16 roundings of 2^-24 on each factor of a rotation, its two products and sum three more
    # (2^-18 of the two factors covers 2.5 times that); FP32's smallest step below
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size + 1e-40).all()


def qkv_rows(n, hq, hkv, dtype, seed, gap=0):
    x = torch.randn((n, (hq + 2 * hkv) * 128 + gap), generator=torch.Generator().manual_seed(seed)) * 3
    x = x.to(dtype)
    return x.cuda()[:, :(hq + 2 * hkv) * 128], x.float().numpy()[:, :(hq + 2 * hkv) * 128].reshape(n, hq + 2 * hkv, 128)


def run_norm(n, hq, hkv, dtype, fmt=None, rotary=128, inter=False, norm=(True, True), k_out=True, layout=0, gap=0, eps=1e-6, seed=0, slots=None, pages=None):
    pages = pages or n // 16 + 3
    cache, raw, bufs = make_cache(hma.HMA_KV_BFP8 if fmt is None else fmt, hkv, pages, hq=hq, key_layout=layout)
    qkv, x = qkv_rows(n, hq, hkv, dtype, seed, gap)
    w = [torch.randn(128, generator=torch.Generator().manual_seed(seed + 9 + i)).to(dtype).cuda() if norm[i] else None for i in (0, 1)]
    table = hma.hma_rope_table(1e6 ** (-np.arange(rotary // 2) / (rotary // 2)), 500) if rotary else None
    pos = rng0(seed).integers(0, 500, n).astype(np.int32)
    q = torch.full((n + 1, hq, 128), 7.5, dtype=torch.bfloat16, device="cuda")
    k = torch.full((n + 1, hkv, 128), 7.5, dtype=torch.bfloat16, device="cuda") if k_out else None
    slots = None if fmt is None else slots if slots is not None else rng0(seed + 1).permutation(pages * 16)[:n]
    hma.hma_qk_norm_rope(cache, 0, qkv, *w, eps, table, None if table is None else torch.from_numpy(pos).cuda(), q[:n], k_out=k[:n] if k_out else None,
                         slots=None if slots is None else torch.from_numpy(np.asarray(slots, np.int64)).cuda(), interleaved=inter)
    torch.cuda.synchronize()
    t = None if table is None else table.cpu().numpy()
    wn = [None if u is None else u.float().cpu().numpy() for u in w]
    assert_rows(q[:n].double().cpu().numpy(), *norm_rope_oracle(x[:, :hq], wn[0], eps, t, pos, inter))
    assert bool((q[n:] == 7.5).all())
    if k_out:
        assert_rows(k[:n].double().cpu().numpy(), *norm_rope_oracle(x[:, hq:hq + hkv], wn[1], eps, t, pos, inter))
        assert bool((k[n:] == 7.5).all())
    return cache, raw, bufs, x, k, slots, qkv


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,hq,hkv,rotary,inter,norm,gap", [
    (1, 1, 1, 128, False, (True, True), 0), (3, 8, 8, 128, True, (True, True), 8), (17, 5, 1, 64, False, (True, False), 0), (33, 40, 8, 16, False, (False, True), 24),
    (5, 12, 4, 96, True, (False, False), 0), (50, 6, 2, 0, False, (True, True), 0), (500, 40, 8, 128, False, (True, True), 8), (1001, 18, 3, 112, True, (True, True), 0),
    (700, 29, 29, 32, False, (True, False), 0), (4, 64, 64, 128, False, (True, True), 0)])
def test_norm_rope_rows(dtype, n, hq, hkv, rotary, inter, norm, gap):
    cache, raw, bufs, *_ = run_norm(n, hq, hkv, dtype, None, rotary, inter, norm, True, gap=gap, seed=n)
    assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0]) and hma.hma_error_flags(cache) == 0        # no slots: nothing cached


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,hq,hkv,layout,kind", [(1, 8, 1, 0, "one"), (37, 10, 2, 1, "scattered"), (70, 9, 3, 0, "late start"), (1003, 40, 8, 0, "in order"), (64, 2, 2, 1, "padded"), (33, 4, 1, 0, "bad")])
def test_norm_rope_fills_the_cache(fmt, dtype, n, hq, hkv, layout, kind):
    pages = n // 16 + 5
    slots = np.array(list(SLOTS[kind](n, pages, rng0(n))), np.int64)
    cache, raw, bufs, x, k, slots, _ = run_norm(n, hq, hkv, dtype, fmt, 64, False, layout=layout, seed=n, slots=slots, pages=pages)
    # the cached key is the BF16 value that k_out shows, exactly; values pass from the input's own type
    flags = records.write(raw[0], cache.desc, slots, k[:n].float().cpu().numpy(), x[:, hq + hkv:])
    assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0]) and bool((bufs[0][-256:] == 0x3C).all())
    assert hma.hma_error_flags(cache) == flags


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_without_k_out_the_cache_is_the_same(fmt):
    slots = np.arange(5, 5 + 100)
    a = run_norm(100, 8, 2, torch.bfloat16, fmt, 128, False, k_out=True, seed=4, slots=slots, pages=9)
    b = run_norm(100, 8, 2, torch.bfloat16, fmt, 128, False, k_out=False, seed=4, slots=slots, pages=9)
    assert torch.equal(a[2][0], b[2][0])


@pytest.mark.gpu
def test_positions_outside_the_table_are_flagged():
    cache, raw, bufs = make_cache(hma.HMA_KV_BFP8, 1, 2, hq=2)
    qkv, x = qkv_rows(4, 2, 1, torch.float32, 1)
    table = hma.hma_rope_table([1.0] * 8, 10)
    q, k = torch.zeros((4, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 1, 128), dtype=torch.bfloat16, device="cuda")
    pos = np.array([3, -1, 10, 9], np.int32)
    hma.hma_qk_norm_rope(cache, 0, qkv, None, None, 0.0, table, torch.from_numpy(pos).cuda(), q, k_out=k)
    assert hma.hma_error_flags(cache) == hma.HMA_FLAG_BAD_POSITION
    pos[1] = pos[2] = 0
    assert_rows(q.double().cpu().numpy(), *norm_rope_oracle(x[:, :2], None, 0.0, table.cpu().numpy(), pos, False))


@pytest.mark.gpu
def test_norm_of_extreme_rows():
    """Rows of zeros, of tiny and of huge numbers; one that holds NaN and Inf leaves the others alone."""
    cache, raw, bufs = make_cache(hma.HMA_KV_BF16, 1, 2, hq=1)
    x = torch.ones((5, 3 * 128))
    x[0] = 0
    x[1] *= 1e-10
    x[2] *= 1e18
    x[3, 0], x[3, 1] = float("nan"), float("inf")
    q, k = torch.zeros((5, 1, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((5, 1, 128), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, device="cuda")
    hma.hma_qk_norm_rope(cache, 0, x.cuda(), w, w, 1e-30, None, None, q, k_out=k)
    got = q.double().cpu().numpy()
    assert (got[0] == 0).all() and (got[[1, 2, 4]] == 1.0).all() and np.isnan(got[3]).all()


@pytest.mark.gpu
def test_an_unrotated_channel_passes_infinities():
    cache, raw, bufs = make_cache(hma.HMA_KV_BF16, 1, 2, hq=1)
    x = torch.ones((1, 3 * 128))
    x[0, 100] = float("inf")
    q, k = torch.zeros((1, 1, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 1, 128), dtype=torch.bfloat16, device="cuda")
    hma.hma_qk_norm_rope(cache, 0, x.cuda(), None, None, 0.0, hma.hma_rope_table([0.5] * 16, 3), torch.tensor([2], dtype=torch.int32, device="cuda"), q, k_out=k)
    got = q.float().cpu()[0, 0]
    assert got[100] == float("inf") and torch.isfinite(got[:100]).all() and (got[101:] == 1).all()


# ---------------------------------------------------------------- refusals
def test_refusals_without_a_gpu():
    L = hma.lib()
    assert L.hma_kv_append(None, 0, None, None, 0, 128, 128, None, 1, None) == hma.HMA_ERR_INVALID_ARG
    assert L.hma_qk_norm_rope(None, 0, None, 0, 384, 1, None, None, 1e-6, None, 0, 0, 0, None, None, None, None, None) == hma.HMA_ERR_INVALID_ARG

    class Fake:
        desc, handle = hma.make_desc(1, 8, 8, 4), None
    t = torch.zeros((2, 8, 128))
    with pytest.raises(hma.HmaError):
        hma.hma_kv_append(Fake, 0, t, t, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(hma.HmaError):
        hma.hma_qk_norm_rope(Fake, 0, t.flatten(1), None, None, 0.0, None, None, t)


@pytest.mark.gpu
def test_refusals():
    cache, raw, bufs = make_cache(hma.HMA_KV_BFP8, 2, 4, hq=4)
    k = torch.zeros((3, 2, 128), device="cuda")
    s = torch.arange(3, device="cuda")
    n0 = hma.hma_launch_count()
    for kk, vv, ss in ((k.half(), k.half(), s), (k, k.bfloat16(), s), (k[:2], k, s), (k, k, s.int()), (k[..., :64], k[..., :64], s), (k.transpose(0, 1), k, s), (k, k, s.cpu())):
        with pytest.raises(hma.HmaError) as e:
            hma.hma_kv_append(cache, 0, kk, vv, ss)
        assert e.value.status == hma.HMA_ERR_INVALID_ARG
    L, p, h = hma.lib(), k.data_ptr(), cache.handle
    ap = lambda layer=0, kp=p, vp=p, dt=1, ks=256, vs=256, sp=s.data_ptr(), n=3: L.hma_kv_append(h, layer, kp, vp, dt, ks, vs, sp, n, None)
    assert [ap(layer=1), ap(layer=-1), ap(kp=None), ap(sp=None), ap(dt=2), ap(ks=255), ap(vs=0), ap(n=-1)] == [1] * 8
    assert [ap(kp=p + 8), ap(ks=258, dt=0), ap(vs=257)] == [3] * 3
    assert [ap(n=(1 << 24) + 1), ap(ks=(1 << 30) + 4)] == [2] * 2 and ap(n=0, kp=None, sp=None) == 0
    qkv = torch.zeros((3, 8 * 128), device="cuda")
    o = torch.zeros((3, 4, 128), dtype=torch.bfloat16, device="cuda")
    tb, po = torch.zeros((4, 32), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    nr = lambda layer=0, x=qkv.data_ptr(), dt=1, st=1024, n=3, wq=None, eps=1e-6, t=tb.data_ptr(), r=4, rot=32, il=0, ps=po.data_ptr(), sl=s.data_ptr(), q=o.data_ptr(), ko=None: \
        L.hma_qk_norm_rope(h, layer, x, dt, st, n, wq, wq, eps, t, r, rot, il, ps, sl, q, ko, None)
    assert [nr(layer=1), nr(x=None), nr(dt=3), nr(st=1020), nr(n=-1), nr(eps=-1.0), nr(eps=float("nan")), nr(t=None), nr(r=0), nr(il=2), nr(ps=None), nr(q=None), nr(sl=None)] == [1] * 13
    assert [nr(rot=8), nr(rot=144), nr(rot=-16), nr(n=(1 << 24) + 1)] == [2] * 4
    assert [nr(x=qkv.data_ptr() + 4), nr(st=1026), nr(wq=tb.data_ptr() + 4), nr(q=o.data_ptr() + 2), nr(ko=o.data_ptr() + 8)] == [3] * 5
    assert nr(n=0, x=None) == 0 and hma.hma_launch_count() == n0
    for bad in (dict(qkv=qkv[:, :1000]), dict(positions=po[:2]), dict(q_out=o[:2]), dict(positions=po.long())):
        args = dict(qkv=qkv, q_weight=None, k_weight=None, eps=0.0, rope_table=tb, positions=po, q_out=o, slots=s)
        args.update(bad)
        with pytest.raises(hma.HmaError):
            hma.hma_qk_norm_rope(cache, 0, **args)


@pytest.mark.gpu
def test_a_four_bit_cache_is_refused_where_it_has_no_meaning():
    cache, raw, bufs = make_cache(hma.HMA_KV_BFP4, 2, 4)
    t = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p, h, L = t.data_ptr(), cache.handle, hma.lib()
    one = lambda: (ctypes.c_void_p * 1)(p)
    i1 = lambda v: (ctypes.c_int32 * 1)(v)
    got = [L.hma_kv_ingest_layer(h, 0, p, p, w, 0, 2, p, 0, 16, None) for w in (0, 1)]
    got += [L.hma_kv_ingest_layer_shards(h, 0, 1, one(), one(), 0, i1(0), i1(2), p, 0, 16, None), L.hma_kv_ingest_request_shards(h, 1, one(), one(), 16, 0, i1(0), i1(2), p, 0, 16, None),
            L.hma_bfp8_dequant_bf16(h, 0, 0, p, 0, 16, p, None), L.hma_bfp8_rebuild_request(h, p, 0, 16, p, None), L.hma_bfp8_dequant_bf16_naive(h, 0, 0, p, 0, 16, p, None)]
    assert got == [hma.HMA_ERR_UNSUPPORTED_SHAPE] * len(got)
    assert L.hma_kv_ingest_layer(h, 0, p, p, 2, 0, 2, p, 0, 16, None) != 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lead", [0, 5, 16])
@pytest.mark.parametrize("hkv,filled", [(2, 1), (64, 9)])
def test_whole_pages_of_slots_at_the_end_of_the_range(fmt, lead, hkv, filled):
    """Sixteen slots in a row from a multiple of 16, as a page has them, up to the largest number there is: skipped and flagged like any other."""
    P, top = 12, 2 ** 63
    runs = [list(range(top - 16, top)), list(range(16 * 3, 16 * 4)), list(range(top - 32, top - 16)), list(range(2 ** 62, 2 ** 62 + 16)), list(range(16 * P, 16 * P + 16))]
    runs += [list(range(16 * p, 16 * p + 16)) for p in range(4, 4 + filled - 1)]
    slots = np.array([-1] * lead + [s for r in runs for s in r], np.int64)
    n = len(slots)
    cache, raw, bufs = make_cache(fmt, hkv, P)
    k, kf = rows(n, hkv, torch.float32, n)
    v, vf = rows(n, hkv, torch.float32, n + 1)
    assert records.write(raw[0], cache.desc, slots, kf, vf) == hma.HMA_FLAG_BAD_PAGE_INGEST
    at = torch.from_numpy(slots).cuda()
    hma.hma_kv_append(cache, 0, k.cuda(), v.cuda(), at)
    torch.cuda.synchronize()
    assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0]) and bool((bufs[0][-256:] == 0x3C).all())
    assert hma.hma_error_flags(cache) == hma.HMA_FLAG_BAD_PAGE_INGEST
    qkv = torch.cat([k[:, :hkv], k, v], 1).flatten(1).cuda()                # the same rows, keys rounded to BF16 first
    assert records.write(raw[0], cache.desc, slots, k.bfloat16().float().numpy(), vf) == hma.HMA_FLAG_BAD_PAGE_INGEST
    hma.hma_qk_norm_rope(cache, 0, qkv, None, None, 0.0, None, None, torch.empty(n, hkv, 128, dtype=torch.bfloat16, device="cuda"), slots=at)
    torch.cuda.synchronize()
    assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0]) and bool((bufs[0][-256:] == 0x3C).all())
    assert hma.hma_error_flags(cache) == hma.HMA_FLAG_BAD_PAGE_INGEST


@pytest.mark.gpu
@pytest.mark.parametrize("stride", [0, 7, 2 ** 31, 2 ** 40])
def test_the_stride_of_a_single_token_is_not_looked_at(stride):
    """A row cut out of a large tensor keeps that tensor's strides."""
    hkv = 2
    cache, raw, bufs = make_cache(hma.HMA_KV_BFP8, hkv, 4)
    k, kf = rows(1, hkv, torch.bfloat16, 1)
    v, vf = rows(1, hkv, torch.bfloat16, 2)
    far = lambda x: x.cuda().as_strided(x.shape, (stride,) + x.stride()[1:])
    slots = torch.tensor([21], device="cuda")
    hma.hma_kv_append(cache, 0, far(k), far(v), slots)
    records.write(raw[0], cache.desc, [21], kf, vf)
    assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0])
    q = torch.empty(1, hkv, 128, dtype=torch.bfloat16, device="cuda")
    hma.hma_qk_norm_rope(cache, 0, far(torch.cat([v, v, k], 1).flatten(1)), None, None, 0.0, None, None, q, slots=slots)
    records.write(raw[0], cache.desc, [21], vf, kf)
    assert np.array_equal(bufs[0][:-256].cpu().numpy(), raw[0]) and torch.equal(q.cpu(), v) and hma.hma_error_flags(cache) == 0
