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
