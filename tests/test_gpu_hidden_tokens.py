"""Tokens that one query of a sequence sees and another one does not: whatever they hold, it reaches only the queries that see them."""
import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma
import records
from records import Paged

BFP8, BF16, BFP4 = hma.HMA_KV_BFP8, hma.HMA_KV_BF16, hma.HMA_KV_BFP4
SHORT = [40, 203, 64, 65, 33, 17, 16, 2, 1, 0]                     # a CTA or less to a segment
LONG = [5000, 0, 2999, 300, 4100, 1, 2017]                        # windows that are cut into many warps' shares
POISON = [(BF16, 0x7FC0), (BF16, 0x7F80), (BF16, 0xFF80), (BFP8, 250), (BFP4, 250)]      # NaN, Inf, -Inf; the largest exponent that attention takes


def put(p, layer, b, t, what):
    """Poison in V of token t of sequence b: the BF16 number with these bits, or codes with this exponent.  BF16 keys get it, too."""
    rec = records.records(layer, p.desc)[p.table[b, t // 16]]
    if p.fmt == BF16:
        for part in (0, 1):
            at = records.places(p.fmt, part)[0][t % 16]
            rec[:, at], rec[:, at + 1] = what & 255, what >> 8
    else:
        rec[:, records.exp_places(p.fmt, 1)[t % 16]] = what


def check(p, call, window, sinks, what):
    """One poisoned token a call, at every place that divides the queries of a sequence: the newest tokens (hidden from older queries) and
    those that the window has just left for newer ones."""
    ref, tol = p.reference(window=window, sinks=sinks)
    Q = p.q_len
    places = [("end", i) for i in range(1, Q)] + ([("edge", i) for i in range(Q - 1)] if window else [])
    for kind, i in places:
        layer, hides = p.raw[0].copy(), np.ones((len(p.lens), Q), bool)
        for b, T in enumerate(p.lens.tolist()):
            ends = [T - (Q - 1 - k) for k in range(Q)]
            t = ends[i] - 1 if kind == "end" else ends[i] - window          # the token of query i; the first one of its window
            if 0 <= t < T:
                put(p, layer, b, t, what)
                hides[b] = [t >= e or (window is not None and t < e - window and t >= sinks) for e in ends]
        assert not hides.all()
        p.cache.layers[0].copy_(torch.from_numpy(layer))
        out = torch.full(p.q.shape, 7.0, device="cuda")
        call(out)
        got = out.double().cpu().numpy()
        assert (np.abs(got - ref) <= tol)[hides].all(), (kind, i, np.argwhere(~(np.abs(got - ref) <= tol).all((2, 3)) & hides))
        flags = hma.hma_error_flags(p.cache)                                # (a query that sees NaN keys has no finite sum)
        assert p.fmt == BF16 or flags == 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,what", POISON)
@pytest.mark.parametrize("q_len", [2, 3, 4])
@pytest.mark.parametrize("lens,hkv,window,sinks", [(SHORT, 2, 21, 3), (SHORT, 1, 16, 0), (LONG, 1, 3000, 40)])
def test_window(fmt, what, q_len, lens, hkv, window, sinks):
    p = Paged(lens, hkv * 3, hkv, fmt, seed=q_len, q_len=q_len, window=window, sinks=sinks)
    ws = hma.new_workspace(p.desc, len(lens) * q_len)
    check(p, lambda out: hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, window, sinks, p.scale, ws), window, sinks, what)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,what", POISON)
@pytest.mark.parametrize("q_len", [2, 4])
@pytest.mark.parametrize("lens,hkv", [(SHORT, 2), (LONG, 1)])
@pytest.mark.parametrize("planned", [False, True])
def test_several_query_tokens(fmt, what, q_len, lens, hkv, planned):
    p = Paged(lens, hkv * 3, hkv, fmt, seed=q_len, q_len=q_len)
    ws = hma.new_workspace(p.desc, len(lens) * q_len)
    plan = hma.hma_decode_attention_plan(p.cache, p.tbl, p.ctx, q_len) if planned else None

    def call(out):
        if planned:
            hma.hma_decode_attention_planned(p.cache, 0, p.q, out, p.tbl, p.ctx, p.scale, plan, ws)
        else:
            hma.hma_decode_attention_multi(p.cache, 0, p.q, out, p.tbl, p.ctx, p.scale, ws)
    check(p, call, None, 0, what)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [BFP8, BFP4])
@pytest.mark.parametrize("q_len", [1, 2, 4])
@pytest.mark.parametrize("exps", [(110, 140), (60, 131), (2, 251)])
@pytest.mark.parametrize("lens,hkv,window,sinks", [(SHORT, 2, 21, 3), (LONG, 1, 3000, 40), (SHORT, 2, None, 0), (LONG, 1, None, 0)])
def test_v_blocks_of_very_different_sizes(fmt, q_len, exps, lens, hkv, window, sinks):
    """Every query keeps what its own blocks leave it.  With R the largest exponent of the query's blocks of a channel, weights reach the second
    product as FP16 numbers p * 2^(E - R + 15): a block with E <= R - 30 counts as zero, which takes at most 2^-30 of the largest
    value (the weights' sum being 1) off the result, and a product is rounded by at most 2^-25, 2^-40 of the largest value for each token."""
    p = Paged(lens, hkv * 3, hkv, fmt, seed=q_len + exps[0], q_len=q_len, window=window, sinks=sinks)
    rec, clean = records.records(p.raw[0], p.desc), records.records(p.clean[0], p.desc)
    at = records.exp_places(fmt, 1)
    e = np.random.default_rng(exps[0]).integers(*exps, clean[..., at].shape, dtype=np.uint8)      # [pages][heads][16][8]
    rec[..., at] = np.where(rec[..., at] == 255, 255, e)                    # (255: what no query sees)
    clean[..., at] = e
    p.cache.layers[0].copy_(torch.from_numpy(p.raw[0]))
    ref, tol = p.reference(window=window, sinks=sinks)
    most, low = (127, 133) if fmt == BFP8 else (8, 129)
    for b, T in enumerate(p.lens.tolist()):
        blocks = np.moveaxis(e[p.table[b, :(T + 15) // 16]], 1, 2).reshape(-1, hkv, 8)      # [tokens][heads][8]
        for i in range(q_len):
            end = max(0, T - (q_len - 1 - i))
            t = np.arange(end)
            if window:
                t = t[(t >= end - window) | (t < sinks)]
            if len(t):
                top = np.ldexp(float(most), blocks[t].max(0).astype(np.int64) - low)        # [heads][8]
                tol[b, i] += np.repeat(np.repeat(top, 16, 1), 3, 0) * (2.0 ** -30 + len(t) * 2.0 ** -40) + 2.0 ** -140      # (fp32's subnormals)
    ws, outs = hma.new_workspace(p.desc, len(lens) * q_len), []
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full(p.q.shape, 7.0, dtype=dt, device="cuda")
        if window:
            hma.hma_decode_attention_window(p.cache, 0, p.q, out, p.tbl, p.ctx, window, sinks, p.scale, ws)
        else:
            hma.hma_decode_attention_multi(p.cache, 0, p.q, out, p.tbl, p.ctx, p.scale, ws)
        outs.append(out)
    p.check(*outs, ref, tol)
