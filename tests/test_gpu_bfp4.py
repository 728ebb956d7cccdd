"""Attention over a cache held in 4 bits: every entry point that reads it, against 64-bit attention over the codes' values."""
import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma
from records import Paged
import records

BFP4 = hma.HMA_KV_BFP4


def run(p, call=hma.hma_decode_attention, layer=0):
    ws = hma.new_workspace(p.desc, len(p.lens))
    outs = []
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full((len(p.lens), p.hq, 128), float("nan"), dtype=dt, device="cuda")
        call(p.cache, layer, p.q[:, 0].contiguous(), out, p.tbl, p.ctx, p.scale, ws)
        outs.append(out)
    torch.cuda.synchronize()
    assert int(ws[:1024 * 64 * 4].max()) == 0
    return outs


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,lens", [
    (1, 1, [1]), (8, 8, [0, 1, 2, 15, 16, 17]), (5, 1, [40] * 7), (64, 8, [300, 5, 0, 1000]), (21, 3, [4000, 16, 33]), (32, 4, list(range(70))), (64, 64, [130, 7]), (8, 1, [20000])])
def test_attention(hq, hkv, lens):
    p = Paged(lens, hq, hkv, BFP4, seed=hq + len(lens))
    p.check(*run(p), *p.reference())


@pytest.mark.gpu
@pytest.mark.parametrize("b,hkv,most", [(1, 1, 1800), (9, 2, 800), (40, 4, 500), (74, 4, 250), (148, 1, 1700), (149, 1, 800), (30, 64, 16), (290, 8, 16), (19, 8, 1500)])
def test_small_calls(b, hkv, most):
    """Every number of segments per CTA that the small path knows, and its neighbours beyond it; empty sequences among them."""
    lens = np.random.default_rng(b).integers(0, most + 1, b)
    lens[0], lens[-1] = 0, most
    p = Paged(lens, hkv * 2, hkv, BFP4, seed=b)
    p.check(*run(p), *p.reference())


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,lens", [(1, [8000]), (1, [1025, 0, 3]), (8, [1024] * 4), (8, [4096, 70, 0, 2000]), (5, [2500, 33]), (2, [5000, 1, 16, 4000, 640]), (16, [2048, 512]), (7, [0, 0, 1500])])
def test_few_long_sequences(hkv, lens):
    """Few sequences with long contexts: either side of the limit at which the list takes over, with empty ones among them."""
    p = Paged(lens, hkv * 3, hkv, BFP4, seed=hkv)
    ref, tol = p.reference()
    p.check(*run(p), ref, tol)
    if hkv * len(lens) <= 32:                              # and two query tokens a warp
        m = Paged(lens, hkv * 3, hkv, BFP4, seed=hkv, q_len=2)
        outs, ws = [torch.full(m.q.shape, float("nan"), dtype=dt, device="cuda") for dt in (torch.float32, torch.bfloat16)], hma.new_workspace(m.desc, 2 * len(lens))
        for o in outs:
            hma.hma_decode_attention_multi(m.cache, 0, m.q, o, m.tbl, m.ctx, m.scale, ws)
        m.check(*outs, *m.reference())
        assert int(ws[:1024 * 64 * 4].max()) == 0


@pytest.mark.gpu
def test_flat_weights_over_a_long_context():
    """Scores near zero: the output is a mean of thousands of values, small beside the codes' offset of 8."""
    p = Paged([16000, 9000], 8, 2, BFP4, seed=8, exps=(127, 128))
    p.q = p.q * 0
    p.check(*run(p), *p.reference())


@pytest.mark.gpu
@pytest.mark.parametrize("exps", [(1, 4), (0, 20), (100, 140), (60, 61), (200, 220)])
def test_exponents(exps):
    """Blocks of very different sizes side by side.  V blocks far below the largest one of their channels may vanish; keys are scaled so
    that the scores stay ordinary."""
    p = Paged([100, 31, 500], 8, 2, BFP4, seed=exps[0], exps=(118, 131))
    at = records.exp_places(BFP4, 1).reshape(-1)
    rng = np.random.default_rng(1)
    rec, clean = records.records(p.raw[0], p.desc), records.records(p.clean[0], p.desc)
    e = rng.integers(*exps, clean[..., at].shape, dtype=np.uint8)
    clean[..., at] = e
    rec[..., at] = np.where(rec[..., at] == 255, 255, e)
    p.cache.layers[0].copy_(torch.from_numpy(p.raw[0]))
    ref, tol = p.reference()
    # 2^-39 of the largest block of a (kv head, 16 channels) column is below what a weight can carry; so are FP32's subnormals
    top = 15 * 2.0 ** (exps[1] - 1 - 129.0)
    p.check(*run(p), ref, np.where(tol > 0, tol + top * 2.0 ** -38 + 2.0 ** -140, 0))


@pytest.mark.gpu
def test_exponents_beyond_the_range_are_flagged():
    p = Paged([40], 4, 1, BFP4, exps=(251, 254))
    run(p)
    assert hma.hma_error_flags(p.cache) & hma.HMA_FLAG_EXPONENT_RANGE


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 2, 3, 8])
def test_multi_and_planned(q_len):
    for lens in ([300, 17, 64, 1000, 0, 3], [5, 40, 100], [3000, 17, 0, 1300]):
        p = Paged(lens, 10, 2, BFP4, seed=q_len, q_len=q_len)
        ws = hma.new_workspace(p.desc, len(lens) * q_len)
        outs = [torch.full(p.q.shape, float("nan"), dtype=dt, device="cuda") for dt in (torch.float32, torch.bfloat16) * 2]
        plan = hma.hma_decode_attention_plan(p.cache, p.tbl, p.ctx, q_len=q_len)
        for o in outs[:2]:
            hma.hma_decode_attention_multi(p.cache, 0, p.q, o, p.tbl, p.ctx, p.scale, ws)
        for o in outs[2:]:
            hma.hma_decode_attention_planned(p.cache, 0, p.q, o, p.tbl, p.ctx, p.scale, plan, ws)
        ref, tol = p.reference()
        p.check(outs[0], outs[1], ref, tol)
        p.check(outs[2], outs[3], ref, tol)
        if max(lens) > 2000:                               # (smaller calls split the work differently without a plan)
            assert torch.equal(outs[0], outs[2])


@pytest.mark.gpu
def test_static_and_simple():
    p = Paged([300, 17, 0, 1000], 10, 2, BFP4, seed=5)
    a32, a16 = run(p)
    s = torch.full_like(a32, float("nan"))
    hma.hma_decode_attention_static(p.cache, 0, p.q[:, 0].contiguous(), s, p.tbl, p.ctx, p.scale)
    assert torch.equal(s, a32)
    e = torch.full_like(a32, float("nan"))
    hma.hma_decode_attention_simple(p.cache, 0, p.q[:, 0].contiguous(), e, p.tbl, p.ctx, p.scale)
    ref, tol = p.reference()
    assert (np.abs(e.double().cpu().numpy() - ref[:, 0]) <= tol[:, 0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("planned", [False, True])
def test_four_bit_prefix_and_bf16_tail(planned):
    """Two caches under one softmax, a 4-bit one first (and, the other way round, as the tail)."""
    a = Paged([300, 0, 17, 1000, 33], 8, 2, BFP4, seed=1)
    b = Paged([20, 40, 0, 5, 0], 8, 2, hma.HMA_KV_BF16, seed=2)
    for first, second in ((a, b), (b, a)):
        both = [torch.full((5, 8, 128), float("nan"), dtype=dt, device="cuda") for dt in (torch.float32, torch.bfloat16)]
        q, ws = a.q[:, 0].contiguous(), hma.new_workspace(a.desc, 5, copies=2)
        for o in both:
            args = [first.cache, second.cache, 0, q, o, first.tbl, first.ctx, second.tbl, second.ctx, a.scale]
            if planned:
                plans = [hma.hma_decode_attention_plan(x.cache, x.tbl, x.ctx) for x in (first, second)]
                hma.hma_decode_attention_mixed_planned(*args, *plans, ws)
            else:
                hma.hma_decode_attention_mixed(*args, ws)
        got = both[0].double().cpu().numpy()
        assert torch.equal(both[1], both[0].bfloat16())
        # the bound of one cache holds for both: weights with 11 bits (one more rounding where the two sums meet), scores to fp32
        qn = q.double().cpu().numpy()
        for s in range(5):
            kv = [records.read(x.clean[0], x.desc, x.table[s, :(int(x.lens[s]) + 15) // 16]) for x in (a, b)]
            k, v = (np.concatenate([kv[i][w][:int(x.lens[s])] for i, x in enumerate((a, b))]) for w in (0, 1))
            for h in range(8):
                sc = qn[s, h] @ k[:, h // 4].T * a.scale
                w = np.exp(sc - sc.max())
                w /= w.sum()
                slip = 2.0 ** -19 * 15 * (np.abs(qn[s, h]).sum() * np.abs(k[:, h // 4]).max() * a.scale)
                assert (np.abs(got[s, h] - w @ v[:, h // 4]) <= (2.0 ** -10 + 2 * slip) * (w @ np.abs(v[:, h // 4]))).all()
    assert hma.hma_error_flags(a.cache) == 0 and hma.hma_error_flags(b.cache) == 0


@pytest.mark.gpu
def test_interleaved_keys_and_other_layers():
    p = Paged([100, 31], 8, 2, BFP4, seed=6, key_layout=1, layers=3)
    for layer in (2, 0):
        p.check(*run(p, layer=layer), *p.reference(layer=layer))


@pytest.mark.gpu
def test_probes_refuse_it():
    p = Paged([100], 8, 2, BFP4)
    ws = hma.new_workspace(p.desc, 1)
    for probe in (hma.hma_kv_read_probe, hma.hma_attention_alu_probe):
        with pytest.raises(hma.HmaError) as e:
            probe(p.cache, 0, p.tbl, p.ctx, ws)
        assert e.value.status == hma.HMA_ERR_UNSUPPORTED_SHAPE


@pytest.mark.gpu
def test_a_plan_of_another_format_is_refused():
    p, r = Paged([100], 8, 2, BFP4), Paged([100], 8, 2, hma.HMA_KV_BFP8)
    plan = hma.hma_decode_attention_plan(r.cache, r.tbl, r.ctx)
    out = torch.full((1, 8, 128), 7.0, device="cuda")
    hma.hma_decode_attention_planned(p.cache, 0, p.q[:, 0].contiguous(), out, p.tbl, p.ctx, p.scale, plan, hma.new_workspace(p.desc, 1))
    assert hma.hma_error_flags(p.cache) == hma.HMA_FLAG_BAD_PLAN and bool((out == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("before,after,good", [(33, 48, True), (48, 49, False), (16, 17, False), (32, 33, False), (64, 33, False), (49, 48, False), (0, 1, False)])
def test_a_plan_lasts_while_the_pages_stay(before, after, good):
    """Entries of the work list hold two pages: a sequence that starts the second page of its last entry is noticed all the same."""
    p = Paged([200, 64, 90], 8, 2, BFP4, seed=3)
    ctx = torch.tensor([200, before, 90], dtype=torch.int32, device="cuda")
    plan = hma.hma_decode_attention_plan(p.cache, p.tbl, ctx)
    ctx[1] = after
    out = torch.zeros((3, 8, 128), device="cuda")
    hma.hma_decode_attention_planned(p.cache, 0, p.q[:, 0].contiguous(), out, p.tbl, ctx, p.scale, plan, hma.new_workspace(p.desc, 3))
    assert hma.hma_error_flags(p.cache) == (0 if good else hma.HMA_FLAG_BAD_PLAN)
    p.lens[1] = after
    ref, tol = p.reference()
    for b in (0, 1, 2) if good else (0, 2):
        assert (np.abs(out[b].double().cpu().numpy() - ref[b, 0]) <= tol[b, 0]).all()


@pytest.mark.gpu
def test_bad_pages_are_skipped_and_flagged():
    p = Paged([100, 100, 40], 4, 1, BFP4, seed=2)
    ref, tol = p.reference()
    for col in (0, 1, 6):
        t = p.tbl.clone()
        t[0, col] = -1
        out = torch.zeros((3, 4, 128), device="cuda")
        hma.hma_decode_attention(p.cache, 0, p.q[:, 0].contiguous(), out, t, p.ctx, p.scale, hma.new_workspace(p.desc, 3))
        assert hma.hma_error_flags(p.cache) == hma.HMA_FLAG_BAD_PAGE_ATTENTION
        assert (np.abs(out[1:].double().cpu().numpy() - ref[1:, 0]) <= tol[1:, 0]).all() and bool(torch.isfinite(out).all())
    t.fill_(-1)                                            # nothing there at all
    hma.hma_decode_attention(p.cache, 0, p.q[:, 0].contiguous(), out, t, p.ctx, p.scale, hma.new_workspace(p.desc, 3))
    assert hma.hma_error_flags(p.cache) == hma.HMA_FLAG_BAD_PAGE_ATTENTION and bool((out == 0).all())


def test_layer_bytes():
    assert hma.hma_cache_layer_bytes(hma.make_desc(2, 32, 8, 100, BFP4)) == 100 * 8 * 2304
    assert hma.hma_cache_layer_bytes(hma.make_desc(2, 32, 8, 100, 3)) == 0
