"""Pages beyond 4 GB of a layer, and calls with nothing to do."""
import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma
from records import HALF

HKV, HQ = 8, 16


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [hma.HMA_KV_BFP8, hma.HMA_KV_BFP4, hma.HMA_KV_BF16])
def test_far_pages_behave_like_near_ones(fmt):
    """The same tokens in the first pages of a small cache and in the last ones of a layer of 5 GB: same bytes, same attention."""
    lens, pages = [70, 0, 300, 17], 40
    far = 5 * 2 ** 30 // (2 * HALF[fmt] * HKV)
    npg = [(n + 15) // 16 for n in lens]
    ids = np.random.default_rng(1).permutation(pages)[:sum(npg)]
    table = np.full((4, 20), -1, np.int64)
    o = 0
    for b, n in enumerate(npg):
        table[b, :n] = ids[o:o + n]
        o += n
    slots = np.concatenate([[table[b, t // 16] * 16 + t % 16 for t in range(n)] for b, n in enumerate(lens)]).astype(np.int64)
    n = len(slots)
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn((n, (HQ + 2 * HKV) * 128), generator=g).bfloat16().cuda()
    w, q, ctx = torch.ones(128, dtype=torch.bfloat16, device="cuda"), torch.empty((n, HQ, 128), dtype=torch.bfloat16, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = []
    for shift, total in ((0, pages), (far - pages, far)):
        cache = hma.KVCache(hma.make_desc(1, HQ, HKV, total, fmt))
        tail = cache.layers[0][-pages * 2 * HALF[fmt] * HKV:]
        tail.fill_(0x11)
        s = torch.from_numpy(slots + 16 * shift).cuda()
        t = torch.from_numpy(np.where(table >= 0, table + shift, -1).astype(np.int32)).cuda()
        hma.hma_qk_norm_rope(cache, 0, qkv, w, w, 1e-6, None, None, q, slots=s)
        k = qkv[: n // 2, HQ * 128:(HQ + HKV) * 128].unflatten(1, (HKV, 128))
        hma.hma_kv_append(cache, 0, k, k, s[: n // 2].contiguous())
        outs = []
        ws = hma.new_workspace(cache.desc, 4)
        for call in (lambda o: hma.hma_decode_attention(cache, 0, q[:4], o, t, ctx, 0.1, ws), lambda o: hma.hma_decode_attention_window(cache, 0, q[:4], o, t, ctx, 50, 3, 0.1, ws),
                     lambda o: hma.hma_decode_attention_simple(cache, 0, q[:4], o, t, ctx, 0.1)):
            out = torch.empty((4, HQ, 128), device="cuda")
            call(out)
            outs.append(out)
        assert hma.hma_error_flags(cache) == 0
        got.append((tail.clone(), outs))
        del cache, tail
    assert torch.equal(got[0][0], got[1][0])
    for a, b in zip(got[0][1], got[1][1]):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all()) and float(a.abs().max()) > 0
    assert float((got[0][1][0] - got[0][1][2]).abs().max()) <= 1e-2


@pytest.mark.gpu
def test_nothing_to_do():
    cache = hma.KVCache(hma.make_desc(1, HQ, HKV, 4), fill=7)
    z = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="cuda")
    starts, pos, slots, left = z(1) + 5, z(3) + 5, z(3, dtype=torch.int64) + 5, z(1) + 4
    hma.hma_step_tables(cache, z(0), z(0), z(0, 2), z(4), left, z(0), starts, pos, slots)
    assert starts.tolist() == [0] and pos.tolist() == [0] * 3 and slots.tolist() == [-1] * 3 and left.tolist() == [4]
    hma.hma_step_tables(cache, z(2), z(2), z(2, 2), z(4), left, z(2), z(3), z(0), z(0, dtype=torch.int64))
    assert left.tolist() == [4]
    n0 = hma.hma_launch_count()
    hma.hma_release_pages(cache, z(0), z(0), z(0, 2), z(4), left)
    rows = z(0, HKV, 128, dtype=torch.bfloat16)
    hma.hma_kv_append(cache, 0, rows, rows, z(0, dtype=torch.int64))
    hma.hma_qk_norm_rope(cache, 0, z(0, (HQ + 2 * HKV) * 128, dtype=torch.bfloat16), None, None, 0.0, None, None, z(0, HQ, 128, dtype=torch.bfloat16), slots=z(0, dtype=torch.int64))
    q = z(0, HQ, 128, dtype=torch.bfloat16)
    hma.hma_decode_attention_window(cache, 0, q, q.clone(), z(0, 2), z(0), 4, 0, 1.0, hma.new_workspace(cache.desc, 1))
    assert hma.hma_launch_count() == n0 and hma.hma_error_flags(cache) == 0 and bool((cache.layers[0] == 7).all())
    # a table of no columns: every sequence is empty
    out = torch.full((2, HQ, 128), 3.0, device="cuda")
    for call in (lambda: hma.hma_decode_attention_window(cache, 0, z(2, HQ, 128, dtype=torch.bfloat16), out, torch.zeros((2, 0), dtype=torch.int32, device="cuda"), z(2) + 9, 4, 2, 1.0, hma.new_workspace(cache.desc, 2)),):
        try:
            call()
        except hma.HmaError as e:                       # an empty table has no address
            assert e.status == hma.HMA_ERR_INVALID_ARG
        else:
            assert bool((out == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [hma.HMA_KV_BFP8, hma.HMA_KV_BFP4, hma.HMA_KV_BF16])
@pytest.mark.parametrize("q_len", [1, 2])
def test_a_table_of_no_columns(fmt, q_len):
    """Every sequence is empty, whatever its length says: rows of zeros, and the table's address is not used.  The binding refuses such a
    tensor (it has no address)."""
    cache = hma.KVCache(hma.make_desc(1, 4, 2, 3, fmt), fill=255)
    q = torch.ones(2, q_len, 4, 128, dtype=torch.bfloat16, device="cuda")
    lens, ws = torch.tensor([9, 0], dtype=torch.int32, device="cuda"), hma.new_workspace(cache.desc, 2 * q_len)
    L, p, end = hma.lib(), lambda t: t.data_ptr(), (ws.data_ptr(), ws.numel(), None)
    calls = {"window": lambda out: L.hma_decode_attention_window(cache.handle, 0, p(q), p(out), 1, p(lens), 0, p(lens), 2, q_len, 4, 2, 1.0, *end),
             "multi": lambda out: L.hma_decode_attention_multi(cache.handle, 0, p(q), p(out), 1, p(lens), 0, p(lens), 2, q_len, 1.0, *end)}
    for name, call in calls.items():
        out = torch.full(q.shape, 3.0, device="cuda")
        assert call(out) == hma.HMA_OK
        torch.cuda.synchronize()
        assert bool((out == 0).all()), name
    assert hma.hma_error_flags(cache) == 0
    empty, out = torch.zeros((2, 0), dtype=torch.int32, device="cuda"), torch.full(q.shape, 3.0, device="cuda")
    for call in (lambda: hma.hma_decode_attention_window(cache, 0, q, out, empty, lens, 4, 2, 1.0, ws), lambda: hma.hma_decode_attention_multi(cache, 0, q, out, empty, lens, 1.0, ws)):
        with pytest.raises(hma.HmaError) as e:
            call()
        assert e.value.status == hma.HMA_ERR_INVALID_ARG and bool((out == 3).all())
