"""The operators of a decode step around paged attention: what is measured, in their plain form and through the library.

    tables      page tables, positions and slots of a step's new tokens from the request lengths
    norm_rope   RMS norm of each query and key head and the rotation, keys and values into a BF16 cache
    append      K/V rows encoded into the records of a BFP8 or BFP4 cache
    window      decode attention over a sliding window and the first tokens
    attention4  decode attention over a cache of 4-bit codes

A cache layer is bytes [page][kv head][record]; a record holds 16 tokens x 128 channels of K, then of V.
"""
import functools
import math

import torch

own = False

D, PT = 128, 16                       # head dim, tokens of a page
HALF = {"bfp8": 2176, "bfp4": 1152, "bf16": 4096}     # bytes of the K (or V) part of a record


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a mid-sized batch: every sequence gets one token, a few start a new page
        dict(name="tables-decode-b32", op="tables", batch=32, median=2048, chunks=0, chunk=0, max_pages=512, pad=32),
        # a mixed step: many decoding sequences and a few prompts in chunks, in a token buffer of fixed size
        dict(name="tables-mixed-b256", op="tables", batch=256, median=4096, chunks=16, chunk=2047, max_pages=2048, pad=40000),
        # latency: the smallest decode batch, fused into the cache of generated tokens
        dict(name="norm-decode-b4", op="norm_rope", tokens=4, hq=32, hkv=8, dtype="bf16", rotary=128, pairs="half", far=4096, cache=True, k_out=False, norm=True),
        # a large decode batch whose projection stays in FP32, partial rotation of neighbouring pairs, far positions
        dict(name="norm-decode-b255-f32", op="norm_rope", tokens=255, hq=64, hkv=8, dtype="f32", rotary=64, pairs="inter", far=131072, cache=True, k_out=True, norm=True),
        # the prompt of one request: no cache, the keys go to a prefill attention
        dict(name="norm-prefill-8192", op="norm_rope", tokens=8192, hq=64, hkv=8, dtype="bf16", rotary=128, pairs="half", far=8192, cache=False, k_out=True, norm=True),
        # a batch of ragged chunks (first and last pages shared with what is cached already) into the 8-bit cache
        dict(name="append8-ragged-1021", op="append", fmt="bfp8", seqs=37, tokens=1021, hkv=8, dtype="f32"),
        # a whole prompt into the 4-bit cache
        dict(name="append4-prompt-8192", op="append", fmt="bfp4", seqs=1, tokens=8192, hkv=8, dtype="bf16"),
        # short window on a small batch: latency
        dict(name="window-b4-w256", op="window", fmt="bfp8", batch=4, hq=32, hkv=8, median=1024, sigma=0.0, window=256, sinks=4, q_len=1),
        # ragged batch, two tokens per sequence, 5 query heads per kv head, odd window, BF16 cache
        dict(name="window-b64-w1000-bf16", op="window", fmt="bf16", batch=64, hq=40, hkv=8, median=2048, sigma=0.8, window=1000, sinks=5, q_len=2),
        # long contexts, long window
        dict(name="window-b32-w4096", op="window", fmt="bfp8", batch=32, hq=64, hkv=8, median=8192, sigma=0.0, window=4096, sinks=16, q_len=1),
        # latency on the 4-bit cache
        dict(name="attn4-b4-ctx1k", op="attention4", batch=4, hq=32, hkv=8, median=1024, sigma=0.0),
        # the benchmark's headline batch on the 4-bit cache
        dict(name="attn4-b32-ctx8k", op="attention4", batch=32, hq=64, hkv=8, median=8192, sigma=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["tables", "norm_rope", "append", "window", "attention4"])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.randint(1, 8)
    if op == "tables":
        b = _log(rng, 1, 256)
        chunks = rng.randint(0, min(b, 16))
        chunk = _log(rng, 1, 2047)
        return dict(op=op, batch=b, median=_log(rng, 16, 4096), chunks=chunks, chunk=chunk, max_pages=2048, pad=b + chunks * chunk + rng.randint(0, 500))
    if op == "norm_rope":
        cache = rng.random() < 0.7
        return dict(op=op, tokens=_log(rng, 1, 4096), hq=hq, hkv=hkv, dtype=rng.choice(["bf16", "f32"]), rotary=rng.choice([32, 64, 96, 128]),
                    pairs=rng.choice(["half", "inter"]), far=_log(rng, 4096, 131072), cache=cache, k_out=not cache or rng.random() < 0.5, norm=rng.random() < 0.8)
    if op == "append":
        n = _log(rng, 1, 8192)
        return dict(op=op, fmt=rng.choice(["bfp8", "bfp4"]), seqs=rng.randint(1, min(n, 64)), tokens=n, hkv=hkv, dtype=rng.choice(["bf16", "f32"]))
    b = _log(rng, 1, 32)
    case = dict(op=op, batch=b, hq=hq, hkv=hkv, median=_log(rng, 1, 4096), sigma=rng.choice([0.0, 0.5]))
    if op == "window":
        case.update(fmt=rng.choice(["bfp8", "bfp4", "bf16"]), window=_log(rng, 1, 4096), sinks=rng.choice([0, 1, 4, 16, 33]), q_len=rng.randint(1, 4))
    return case


# ---------------------------------------------------------------- record layouts (positions of the elements of 16 x 128)
@functools.cache
def _layout(fmt, device):
    """Byte offsets inside a record's half, [16][128] each for K and V elements, [16][8] for their exponents; 4-bit codes also
    say whether they sit in the upper half of the byte."""
    tok = torch.arange(PT, device=device)[:, None]
    ch = torch.arange(D, device=device)[None, :]
    j, cb = ch // 16, ch % 16
    b8 = torch.arange(8, device=device)[None, :]
    ke, ve = (tok % 8) * 16 + (tok // 8) * 8 + b8, (tok % 8) // 2 * 32 + b8 * 4 + tok % 2 + 2 * (tok // 8)
    kh = vh = None
    if fmt == "bfp8":
        k = 128 + (tok // 8 + 2 * (j // 4)) * 512 + ((tok % 8) * 4 + cb // 4) * 16 + (j % 4) * 4 + cb % 4
        v = 128 + (j // 2) * 512 + ((cb % 8) * 4 + (tok % 8) // 2) * 16 + ((j % 2) * 2 + cb // 8) * 4 + tok % 2 + 2 * (tok // 8)
    elif fmt == "bfp4":
        k = 128 + (j // 4) * 512 + ((tok % 8) * 4 + cb // 4) * 16 + (j % 4) * 4 + 2 * (cb % 2) + tok // 8
        kh = ((cb // 2) % 2).expand(PT, D)
        v = 128 + (j // 4) * 512 + ((cb % 8) * 4 + (tok % 8) // 2) * 16 + (j % 4) * 4 + 2 * (tok % 2) + tok // 8
        vh = (cb // 8).expand(PT, D)
    else:
        k = (tok // 8 + 2 * (j // 2)) * 512 + ((tok % 8) * 4 + cb // 4) * 16 + (j % 2) * 8 + (cb % 4) * 2
        v = j * 512 + ((cb % 8) * 4 + (tok % 8) // 2) * 16 + (tok // 8 * 2 + cb // 8) * 4 + tok % 2 * 2
    return k.expand(PT, D), v.expand(PT, D), ke, ve, kh, vh


def _encode(x, fmt):
    """fp32 [..., 128] -> exponent bytes [..., 8] and codes [..., 128]: the block's largest exponent field, the significand shifted to
    it and rounded to nearest-even onto 7 (BFP8) or 3 (BFP4) bits, saturating; sign and magnitude (BFP8) or offset by 8 (BFP4)."""
    most, drop = (127, 17) if fmt == "bfp8" else (7, 21)
    bits = x.contiguous().view(torch.int32).reshape(*x.shape[:-1], 8, 16)
    e = (bits >> 23) & 0xFF
    top = e.amax(-1, keepdim=True)
    sig = (bits & 0x7FFFFF) | 0x800000
    sh = (drop + top - e).clamp(max=30)
    m = sig >> sh
    rem, half = sig & ((1 << sh) - 1), 1 << (sh - 1)
    m = m + ((rem > half) | ((rem == half) & ((m & 1) == 1))).int()
    m = torch.where(e == 0, torch.zeros_like(m), m.clamp(max=most))
    neg = bits < 0
    code = m | (neg.int() << 7) if fmt == "bfp8" else torch.where(neg, 8 - m, 8 + m)
    return top.squeeze(-1).to(torch.uint8), code.reshape(x.shape).to(torch.uint8)


def _write(layer, fmt, pages, toks, heads, k, v):
    """Rows k, v [n][heads][128] (fp32, or bf16 for a BF16 cache) into the records of `layer` at (pages[n], toks[n])."""
    kb, vb, ke, ve, kh, vh = _layout(fmt, layer.device)
    half = HALF[fmt]
    rec = ((pages[:, None] * heads + torch.arange(heads, device=layer.device)) * (2 * half))[..., None]       # [n][heads][1]
    for x, off, eoff, hi, base in ((k, kb, ke, kh, 0), (v, vb, ve, vh, half)):
        at = rec + base + off[toks][:, None, :]
        if fmt == "bf16":
            layer.view(torch.bfloat16)[at // 2] = x
            continue
        e, code = _encode(x, fmt)
        layer[rec + base + eoff[toks][:, None, :]] = e
        if fmt == "bfp8":
            layer[at] = code
        else:                     # the two codes of a byte belong to one token: the lower one's channel names the byte
            up = hi[0].bool()
            lower, upper = (~up).nonzero().squeeze(1), up.nonzero().squeeze(1)      # ascending: code i of one meets code i of the other
            layer[at[..., lower]] = code[..., lower] | (code[..., upper] << 4)
    return layer


def _read(records, fmt):
    """Records [..., 2 * HALF] -> K and V values fp32 [..., 16][128]."""
    kb, vb, ke, ve, kh, vh = _layout(fmt, records.device)
    half = HALF[fmt]
    got = []
    for off, eoff, hi, base in ((kb, ke, kh, 0), (vb, ve, vh, half)):
        if fmt == "bf16":
            got.append(records.view(torch.bfloat16)[..., (base + off).reshape(-1) // 2].reshape(*records.shape[:-1], PT, D).float())
            continue
        b = records[..., (base + off).reshape(-1)].reshape(*records.shape[:-1], PT, D).int()
        e = records[..., (base + eoff).reshape(-1)].reshape(*records.shape[:-1], PT, 8).int().repeat_interleave(16, -1)
        if fmt == "bfp8":
            m = torch.where(b >= 128, -(b & 127), b)
            got.append(torch.ldexp(m.float(), e - 133))
        else:
            got.append(torch.ldexp((((b >> (4 * hi)) & 15) - 8).float(), e - 129))
    return got


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lens(median, sigma, batch, most, g):
    t = torch.exp(math.log(median) + sigma * torch.randn(batch, generator=g, device="cuda"))
    return t.round().clamp(1, most).int()


def _filled(pages, hkv, fmt, g):
    """A layer of `pages` pages whose every record holds N(0,1) values, 1 % of the (kv head, channel) pairs 20 times as large."""
    layer = torch.empty(pages * hkv * 2 * HALF[fmt], dtype=torch.uint8, device="cuda")
    big = torch.where(torch.rand((2, hkv, D), generator=g, device="cuda") < 0.01, 20.0, 1.0)
    for p0 in range(0, pages, 2048):
        n = min(2048, pages - p0)
        kv = [torch.randn((n * PT, hkv, D), generator=g, device="cuda") * big[i] for i in (0, 1)]
        if fmt == "bf16":
            kv = [x.bfloat16() for x in kv]
        at = torch.arange(p0 * PT, (p0 + n) * PT, device="cuda")
        _write(layer, fmt, at // PT, at % PT, hkv, *kv)
    return layer


def _paged(lens, g):
    """A block table over randomly placed pages, and the number of pages."""
    npg = (lens.long() + PT - 1) // PT
    most, total = int(npg.max()), int(npg.sum())
    ids = torch.randperm(total, generator=g, device="cuda")
    col = torch.arange(max(most, 1), device="cuda")
    at = (npg.cumsum(0) - npg)[:, None] + col
    return torch.where(col < npg[:, None], ids[at.clamp(max=max(total - 1, 0))], -1).int().contiguous(), max(total, 1)


def prepare(case, seed):
    g, s = _gen(seed), dict(case)
    if case["op"] == "tables":
        B = case["batch"]
        past = _lens(case["median"], 0.8, B, 16 * (case["max_pages"] - 130), g)
        new = torch.ones(B, dtype=torch.int32, device="cuda")
        new[B - case["chunks"]:] = case["chunk"]
        past[B - case["chunks"]:] = past[B - case["chunks"]:] // 2048 * 2048 // 4       # chunks start where earlier chunks ended, or at 0
        held = (past.long() + PT - 1) // PT
        pages = int(held.sum()) + B * 2 + case["chunks"] * (case["chunk"] // PT + 2)
        ids = torch.randperm(pages, generator=g, device="cuda").int()
        col = torch.arange(case["max_pages"], device="cuda")
        at = ((held.cumsum(0) - held)[:, None] + col).clamp(max=pages - 1)
        s["table"] = torch.where(col < held[:, None], ids[at], -1).contiguous()
        s["free"] = torch.cat([ids[int(held.sum()):], ids.new_zeros(int(held.sum()))])
        s["count"] = torch.tensor([pages - int(held.sum())], dtype=torch.int32, device="cuda")
        s["past"], s["new"], s["pages"] = past, new, pages
        for name, n, t in (("ctx", B, torch.int32), ("starts", B + 1, torch.int32), ("positions", case["pad"], torch.int32), ("slots", case["pad"], torch.int64), ("left", 1, torch.int32)):
            s[name] = torch.empty(n, dtype=t, device="cuda")
        return s
    if case["op"] == "norm_rope":
        n, hq, hkv = case["tokens"], case["hq"], case["hkv"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["qkv"] = (torch.randn((n, (hq + 2 * hkv) * D), generator=g, device="cuda") * 3).to(dt)
        s["wq"], s["wk"] = ((1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) for _ in range(2))
        if not case["norm"]:
            s["wq"] = s["wk"] = None
        half = case["rotary"] // 2
        freq = 1e6 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(case["far"], dtype=torch.float64, device="cuda")[:, None] * freq
        s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()       # [position][cos | sin], from 64-bit angles
        if n == case["far"]:
            s["positions"] = torch.arange(n, dtype=torch.int32, device="cuda")
        else:
            s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device="cuda", dtype=torch.int32)
        s["pages"] = max(1, -(-n // PT) * 2)
        s["slots"] = torch.randperm(s["pages"] * PT, generator=g, device="cuda")[:n].contiguous()      # one token of each sequence: anywhere
        if case["cache"]:
            s["layer"] = torch.zeros(s["pages"] * hkv * 2 * HALF["bf16"], dtype=torch.uint8, device="cuda")
        s["q"] = torch.empty((n, hq, D), dtype=torch.bfloat16, device="cuda")
        s["k"] = torch.empty((n, hkv, D), dtype=torch.bfloat16, device="cuda") if case["k_out"] else None
        return s
    if case["op"] == "append":
        n, hkv, S = case["tokens"], case["hkv"], case["seqs"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["k"], s["v"] = (torch.randn((n, hkv, D), generator=g, device="cuda").to(dt) for _ in range(2))
        s["k"][:, :, :: 97] *= 20                       # outlier channels, as keys have them
        cut = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), (torch.randperm(n - 1, generator=g, device="cuda")[: S - 1] + 1).sort().values,
                         torch.full((1,), n, device="cuda")])
        size = cut.diff()
        first = torch.randint(0, 500, (S,), generator=g, device="cuda") if S > 1 else torch.zeros(1, dtype=torch.long, device="cuda")
        npg = (first + size + PT - 1) // PT
        base = npg.cumsum(0) - npg
        s["pages"] = n // PT + 34 * S                   # enough for any of these first positions
        ids = torch.randperm(s["pages"], generator=g, device="cuda")
        seq = torch.repeat_interleave(torch.arange(S, device="cuda"), size)
        pos = first[seq] + torch.arange(n, device="cuda") - cut[seq]
        s["slots"] = (ids[base[seq] + pos // PT] * PT + pos % PT).contiguous()
        s["layer"] = torch.randint(0, 256, (s["pages"] * hkv * 2 * HALF[case["fmt"]],), generator=g, device="cuda", dtype=torch.uint8)
        return s
    fmt = case.get("fmt", "bfp4")
    lens = _lens(case["median"], case["sigma"], case["batch"], 4 * case["median"], g)
    s["table"], s["pages"] = _paged(lens, g)
    s["lens"] = lens
    s["layer"] = _filled(s["pages"], case["hkv"], fmt, g)
    shape = (case["batch"], case["hq"], D) if case["op"] == "attention4" else (case["batch"], case["q_len"], case["hq"], D)
    s["q"] = torch.randn(shape, generator=g, device="cuda").bfloat16()
    s["out"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------- plain forms
def _tables(s):
    B, pad, dev = s["batch"], s["pad"], s["past"].device
    past, end = s["past"].long(), s["past"].long() + s["new"]
    held, want = (past + PT - 1) // PT, (end + PT - 1) // PT
    grow = want - held
    before = grow.cumsum(0) - grow
    col = torch.arange(s["max_pages"], device=dev)
    rank = before[:, None] + col - held[:, None]
    fresh = s["free"][(s["count"].long() - 1 - rank).clamp(0, s["free"].numel() - 1)]
    table = torch.where((col >= held[:, None]) & (col < want[:, None]), fresh, s["table"])
    stop = s["new"].long().cumsum(0)
    starts = torch.cat([stop.new_zeros(1), stop])
    i = torch.arange(pad, device=dev)
    seq = torch.searchsorted(stop, i, right=True).clamp(max=B - 1)
    pos = past[seq] + i - starts[seq]
    there = i < stop[-1]
    page = table[seq, (pos // PT).clamp(max=s["max_pages"] - 1)].long()
    return {"table": table, "context": end.int(), "starts": starts.int(), "positions": torch.where(there, pos, 0).int(),
            "slots": torch.where(there, page * PT + pos % PT, -1), "left": s["count"] - grow.sum().int()}


def _norm_rope(s):
    n, hq, hkv, r = s["tokens"], s["hq"], s["hkv"], s["rotary"]
    x = s["qkv"].view(n, hq + 2 * hkv, D)
    cs = s["rope"][s["positions"].long()][:, None, :]
    cos, sin = cs[..., : r // 2], cs[..., r // 2:]

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        if s["pairs"] == "half":
            a, b = x[..., : r // 2], x[..., r // 2: r]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1).bfloat16()
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1).bfloat16()

    got = {"q": turned(x[:, :hq], s["wq"])}
    k = turned(x[:, hq: hq + hkv], s["wk"])
    if s["k_out"]:
        got["k"] = k
    if s["cache"]:
        got["layer"] = _write(s["layer"], "bf16", s["slots"] // PT, s["slots"] % PT, hkv, k, x[:, hq + hkv:].bfloat16()).view(torch.bfloat16)
    return got


def _append(s):
    return _write(s["layer"], s["fmt"], s["slots"] // PT, s["slots"] % PT, s["hkv"], s["k"].float(), s["v"].float())


def _softmax_sum(q, k, v, seen, hkv):
    """q [rows][hq][128], k and v [rows][tokens][hkv][128], seen [rows][tokens] -> [rows][hq][128]; a row that sees nothing is zeros."""
    R, hq = q.shape[0], q.shape[1]
    score = torch.einsum("rhgd,rthd->rhgt", q.float().view(R, hkv, hq // hkv, D), k) / math.sqrt(D)
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    return torch.einsum("rhgt,rthd->rhgd", p / p.sum(-1, keepdim=True).clamp(min=1e-30), v).reshape(R, hq, D)


def _pages_read(s, table, fmt):
    """The values of the pages that `table` [rows][pages] names, [rows][tokens][hkv][128] of K and of V."""
    rec = s["layer"].view(s["pages"], s["hkv"], 2 * HALF[fmt])[table.clamp(min=0).long()]
    return [x.transpose(2, 3).reshape(table.shape[0], -1, s["hkv"], D) for x in _read(rec, fmt)]


def _attention4(s):
    k, v = _pages_read(s, s["table"], "bfp4")
    seen = torch.arange(k.shape[1], device=k.device) < s["lens"][:, None]
    return _softmax_sum(s["q"], k, v, seen, s["hkv"]).bfloat16()


def _window(s):
    dev, Q, W = s["q"].device, s["q_len"], s["window"]
    upto = (s["lens"].long()[:, None] - (Q - 1) + torch.arange(Q, device=dev)).clamp(min=0).reshape(-1, 1)      # tokens up to the query itself
    head = min(-(-s["sinks"] // PT), s["table"].shape[1])
    first = (upto - W).clamp(min=0) // PT
    col = torch.arange(head + -(-W // PT) + 1, device=dev)
    page = torch.where(col < head, col, first + col - head)
    ok = ((col < head) | (page >= head)) & (page * PT < upto)
    table = s["table"].repeat_interleave(Q, 0).gather(1, torch.where(ok, page, 0))
    t = (page[..., None] * PT + torch.arange(PT, device=dev)).flatten(1)
    seen = ok.repeat_interleave(PT, 1) & (t < upto) & ((t >= upto - W) | (t < s["sinks"]))
    k, v = _pages_read(s, table, s["fmt"])
    return _softmax_sum(s["q"].flatten(0, 1), k, v, seen, s["hkv"]).bfloat16().view_as(s["q"])


# ---------------------------------------------------------------- the library's calls
def _handle(s, fmt):
    """The cache handle over the state's layer and, for attention, its workspace: made by a state's first pass, then kept."""
    from paper_2606_29986_b200 import hma
    if "handle" not in s:
        code = {"bfp8": hma.HMA_KV_BFP8, "bf16": hma.HMA_KV_BF16, "bfp4": getattr(hma, "HMA_KV_BFP4", None)}[fmt]
        desc = hma.make_desc(1, s.get("hq", s.get("hkv", 1)), s.get("hkv", 1), s["pages"], code)
        if "layer" not in s:
            s["unused"] = torch.empty(hma.hma_cache_layer_bytes(desc), dtype=torch.uint8, device="cuda")
        s["handle"] = hma.KVCache(desc, layers=[s["layer"] if "layer" in s else s["unused"]])
        if s["op"] in ("window", "attention4"):
            s["workspace"] = hma.new_workspace(desc, s["batch"] * s.get("q_len", 1))
    return hma, s["handle"]


def run(state):
    s = state
    if not own:
        return {"tables": _tables, "norm_rope": _norm_rope, "append": _append, "window": _window, "attention4": _attention4}[s["op"]](s)
    if s["op"] == "tables":
        hma, cache = _handle(s, "bfp8")
        hma.hma_step_tables(cache, s["past"], s["new"], s["table"], s["free"], s["count"], s["ctx"], s["starts"], s["positions"], s["slots"], s["left"])
        return {"table": s["table"], "context": s["ctx"], "starts": s["starts"], "positions": s["positions"], "slots": s["slots"], "left": s["left"]}
    if s["op"] == "norm_rope":
        hma, cache = _handle(s, "bf16")
        hma.hma_qk_norm_rope(cache, 0, s["qkv"], s["wq"], s["wk"], 1e-6, s["rope"], s["positions"], s["q"], k_out=s["k"],
                             slots=s["slots"] if s["cache"] else None, interleaved=s["pairs"] == "inter")
        got = {"q": s["q"]}
        if s["k_out"]:
            got["k"] = s["k"]
        if s["cache"]:
            got["layer"] = s["layer"].view(torch.bfloat16)
        return got
    if s["op"] == "append":
        hma, cache = _handle(s, s["fmt"])
        hma.hma_kv_append(cache, 0, s["k"], s["v"], s["slots"])
        return s["layer"]
    if s["op"] == "window":
        hma, cache = _handle(s, s["fmt"])
        hma.hma_decode_attention_window(cache, 0, s["q"], s["out"], s["table"], s["lens"], s["window"], s["sinks"], 1 / math.sqrt(D), s["workspace"])
        return s["out"]
    hma, cache = _handle(s, "bfp4")
    hma.hma_decode_attention(cache, 0, s["q"], s["out"], s["table"], s["lens"], 1 / math.sqrt(D), s["workspace"])
    return s["out"]


# ---------------------------------------------------------------- work and 64-bit results
def work(case):
    op = case["op"]
    if op == "tables":
        n = case["batch"] + case["chunks"] * (case["chunk"] - 1)
        grown = case["batch"] // PT + case["chunks"] * (case["chunk"] // PT + 1)
        return {"bytes": 16 * case["batch"] + 8 * grown + 12 * case["pad"], "flops": 4 * n}
    if op == "norm_rope":
        n, hq, hkv, b = case["tokens"], case["hq"], case["hkv"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * (D * b * (hq + hkv * (2 if case["cache"] else 1)) + 4 * case["rotary"] + 4 + 2 * D * (hq + hkv * (bool(case["k_out"]) + 2 * case["cache"]))),
                "flops": n * (hq + hkv) * D * 8}
    if op == "append":
        n, hkv, b = case["tokens"], case["hkv"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * (hkv * (2 * D * b + HALF[case["fmt"]] // 8) + 8), "flops": n * hkv * D * 8}
    fmt = case.get("fmt", "bfp4")
    rows = case["batch"] * case.get("q_len", 1)
    seen = case["median"] * math.exp(case["sigma"] ** 2 / 2)
    cached = seen + 0
    if op == "window":
        seen = min(seen, case["window"] + case["sinks"])
        cached = min(cached, seen + case["q_len"] - 1)
    return {"bytes": case["batch"] * cached * case["hkv"] * HALF[fmt] / 8 + rows * case["hq"] * D * 4, "flops": 4 * rows * seen * case["hq"] * D}


def _element(rec, fmt, what, tok):
    """128 values, in 64 bits, of token `tok` (K: what = 0, V: 1) of records [..., bytes]."""
    c = torch.arange(D, device=rec.device)
    half = rec[..., what * HALF[fmt]: (what + 1) * HALF[fmt]]
    upper, odd, row, blk, c16 = tok // 8, tok % 2, tok % 8, c // 16, c % 16
    if fmt == "bf16":
        if what == 0:
            word = (blk // 2) * 256 * 2 + upper * 256 + (row * 4 + c16 // 4) * 8 + (blk % 2) * 4 + c16 % 4
        else:
            word = blk * 256 + (c16 % 8 * 4 + row // 2) * 8 + (upper * 2 + c16 // 8) * 2 + odd
        return half.contiguous().view(torch.bfloat16)[..., word].double()
    ex = (row * 16 + upper * 8 + blk) if what == 0 else (row // 2 * 32 + blk * 4 + odd + 2 * upper)
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=rec.device), half[..., ex].double() - (133 if fmt == "bfp8" else 129))
    if fmt == "bfp8":
        if what == 0:
            at = 128 + 512 * upper + 1024 * (blk // 4) + 64 * row + 16 * (c16 // 4) + 4 * (blk % 4) + c16 % 4
        else:
            at = 128 + 512 * (blk // 2) + 64 * (c16 % 8) + 16 * (row // 2) + 8 * (blk % 2) + 4 * (c16 // 8) + odd + 2 * upper
        b = half[..., at].double()
        return torch.where(b > 127, 128 - b, b) * power
    if what == 0:
        at, shift = 128 + 512 * (blk // 4) + 64 * row + 16 * (c16 // 4) + 4 * (blk % 4) + 2 * (c16 % 2) + upper, c16 // 2 % 2
    else:
        at, shift = 128 + 512 * (blk // 4) + 64 * (c16 % 8) + 16 * (row // 2) + 4 * (blk % 4) + 2 * odd + upper, c16 // 8
    b = half[..., at].double()
    return (torch.where(shift == 1, torch.floor(b / 16), torch.remainder(b, 16)) - 8) * power


def _exact_attention(case, s):
    fmt, Q = case.get("fmt", "bfp4"), case.get("q_len", 1)
    hkv, hq = case["hkv"], case["hq"]
    layer = s["layer"].view(s["pages"], hkv, 2 * HALF[fmt])
    q = s["q"].double().view(case["batch"], Q, hkv, hq // hkv, D)
    out = torch.zeros_like(q)
    for b, T in enumerate(s["lens"].tolist()):
        rec = layer[s["table"][b, : -(-T // PT)].long()]                                # [pages][hkv][bytes]
        k, v = (torch.stack([_element(rec, fmt, w, t) for t in range(PT)], 2).transpose(1, 2).reshape(-1, hkv, D)[:T] for w in (0, 1))
        for i in range(Q):
            end = T - (Q - 1 - i)
            if end <= 0:
                continue
            t = torch.arange(end, device=k.device)
            if case["op"] == "window":
                t = t[(t >= end - case["window"]) | (t < case["sinks"])]
            a = torch.einsum("hgd,thd->hgt", q[b, i], k[t]) / math.sqrt(D)
            out[b, i] = torch.einsum("hgt,thd->hgd", torch.softmax(a, -1), v[t])
    return out.view(s["q"].shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("window", "attention4"):
        return _exact_attention(case, s)
    if case["op"] == "norm_rope":
        n, hq, hkv, r = case["tokens"], case["hq"], case["hkv"], case["rotary"]
        x = s["qkv"].double().view(n, -1, D)
        freq = torch.pow(torch.tensor(1e6, dtype=torch.float64, device="cuda"), -torch.arange(r // 2, dtype=torch.float64, device="cuda") / (r // 2))
        turn = torch.polar(torch.ones(n, r // 2, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * freq)[:, None]
        got = {}
        for name, part, w in (("q", x[:, :hq], s["wq"]), ("k", x[:, hq: hq + hkv], s["wk"])):
            y = part / torch.sqrt(part.square().sum(-1, keepdim=True) / D + 1e-6) * w.double() if w is not None else part.clone()
            one, two = (slice(0, r // 2), slice(r // 2, r)) if case["pairs"] == "half" else (slice(0, r, 2), slice(1, r, 2))
            z = torch.complex(y[..., one], y[..., two]) * turn
            y[..., one], y[..., two] = z.real, z.imag
            got[name] = y
        v, k = x[:, hq + hkv:], got["k"]
        if not case["k_out"]:
            del got["k"]
        if case["cache"]:
            full = torch.zeros(s["layer"].numel() // 2, dtype=torch.float64, device="cuda")
            c = torch.arange(D, device="cuda")
            for i, at in enumerate(s["slots"].tolist()):
                t, blk, c16 = at % PT, c // 16, c % 16
                kw = (blk // 2) * 512 + t // 8 * 256 + (t % 8 * 4 + c16 // 4) * 8 + (blk % 2) * 4 + c16 % 4
                vw = 2048 + blk * 256 + (c16 % 8 * 4 + t % 8 // 2) * 8 + (t // 8 * 2 + c16 // 8) * 2 + t % 2
                base = (at // PT * hkv + torch.arange(hkv, device="cuda")[:, None]) * 4096
                full[base + kw] = k[i]
                full[base + vw] = v[i]
            got["layer"] = full
        return got
    return None           # whole numbers: the two sides have to be equal
