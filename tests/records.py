"""Records of a cache layer in numpy, straight from the formulas of include/hma.h: encode rows into them, read values out of them."""
import numpy as np

from paper_2606_29986_b200 import hma

HALF = {hma.HMA_KV_BFP8: 2176, hma.HMA_KV_BF16: 4096, hma.HMA_KV_BFP4: 1152}


def bf16_round(x):
    """fp32 array -> bits of the nearest-even BF16 numbers (uint16)."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32)
    r = ((b.astype(np.uint64) + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where((b & 0x7FFFFFFF) > 0x7F800000, np.uint16(0x7FC0), r)


def bf16_value(bits):
    return (np.asarray(bits, np.uint32) << 16).view(np.float32).astype(np.float64)


def encode(x, fmt):
    """fp32 [128] -> (exponent bytes [8], codes [128]); NaN and Inf count as zero."""
    x = np.ascontiguousarray(x, np.float32)
    field = (x.view(np.uint32) >> 23) & 0xFF
    good = (field != 255) & (field != 0)
    E = np.where(good, field, 0).reshape(8, 16).max(1)
    top, most = (133, 127) if fmt == hma.HMA_KV_BFP8 else (129, 7)
    with np.errstate(all="ignore"):
        m = np.rint(np.ldexp(np.where(good, np.abs(x.astype(np.float64)), 0.0), top - np.repeat(E, 16).astype(np.int64)))      # halves to even
    m = np.minimum(m, most).astype(np.int64)
    neg = x.view(np.uint32) >> 31 == 1
    return E.astype(np.uint8), (np.where(neg, m | 128, m) if fmt == hma.HMA_KV_BFP8 else np.where(neg, 8 - m, 8 + m)).astype(np.uint8)


def places(fmt, what):
    """Byte offsets in a record of all elements [16][128], and the nibble they sit in (4-bit) or None."""
    tok, ch = np.meshgrid(np.arange(16), np.arange(128), indexing="ij")
    j, k = ch // 16, tok % 2 + 2 * (tok // 8)
    if fmt == hma.HMA_KV_BFP8:
        if what == 0:
            return 128 + (tok // 8 + 2 * (j // 4)) * 512 + (tok % 8 * 4 + ch % 16 // 4) * 16 + j % 4 * 4 + ch % 4, None
        return 2304 + j // 2 * 512 + (ch % 8 * 4 + tok % 8 // 2) * 16 + (j % 2 * 2 + ch % 16 // 8) * 4 + k, None
    if fmt == hma.HMA_KV_BFP4:
        if what == 0:
            return 128 + j // 4 * 512 + (tok % 8 * 4 + ch % 16 // 4) * 16 + j % 4 * 4 + 2 * (ch % 2) + tok // 8, ch // 2 % 2
        return 1280 + j // 4 * 512 + (ch % 8 * 4 + tok % 8 // 2) * 16 + j % 4 * 4 + 2 * (tok % 2) + tok // 8, ch % 16 // 8
    if what == 0:
        return (tok // 8 + 2 * (j // 2)) * 512 + (tok % 8 * 4 + ch % 16 // 4) * 16 + j % 2 * 8 + ch % 4 * 2, None
    return 4096 + j * 512 + (ch % 8 * 4 + tok % 8 // 2) * 16 + (tok // 8 * 2 + ch % 16 // 8) * 4 + tok % 2 * 2, None


def exp_places(fmt, what):
    """Byte offsets of the exponents [16][8]."""
    tok, j = np.meshgrid(np.arange(16), np.arange(8), indexing="ij")
    if what == 0:
        return tok % 8 * 16 + tok // 8 * 8 + j
    return HALF[fmt] + tok % 8 // 2 * 32 + j * 4 + tok % 2 + 2 * (tok // 8)


def records(layer, desc):
    """A view [pages][kv heads][bytes] of a layer's bytes (numpy)."""
    return layer.reshape(int(desc.num_pages), desc.num_kv_heads, 2 * HALF[desc.format])


def write(layer, desc, slots, k, v):
    """What hma_kv_append does to a layer (numpy uint8, in place); returns the flags it raises.  k, v: fp32 [n][kv heads][128]."""
    fmt, rec, flags = desc.format, records(layer, desc), 0
    order = np.arange(128) if not desc.key_layout else (np.arange(128) >> 1) + 64 * (np.arange(128) & 1)
    for i, s in enumerate(np.asarray(slots).tolist()):
        if s == -1:
            continue
        if s < 0 or s >= desc.num_pages * 16:
            flags |= hma.HMA_FLAG_BAD_PAGE_INGEST
            continue
        page, tok = divmod(s, 16)
        for h in range(desc.num_kv_heads):
            for what, x in ((0, k[i, h][order]), (1, v[i, h])):
                at, nib = places(fmt, what)
                r, at = rec[page, h], at[tok]
                if fmt == hma.HMA_KV_BF16:
                    b = bf16_round(x)
                    r[at], r[at + 1] = b & 255, b >> 8
                    continue
                if not np.isfinite(x).all():
                    flags |= hma.HMA_FLAG_BAD_VALUE_ENCODE
                E, code = encode(x, fmt)
                r[exp_places(fmt, what)[tok]] = E
                if nib is None:
                    r[at] = code
                else:
                    low = nib[tok] == 0
                    r[at[low]] = (r[at[low]] & 0xF0) | code[low]
                    r[at[~low]] = (r[at[~low]] & 0x0F) | (code[~low] << 4)
    return flags


def read(layer, desc, pages, heads=None):
    """float64 values (K, V), each [tokens of `pages` in order][kv heads][128], in the cache's channel order."""
    fmt, rec = desc.format, records(layer, desc)[np.asarray(pages, np.int64)]
    got = []
    for what in (0, 1):
        at, nib = places(fmt, what)
        if fmt == hma.HMA_KV_BF16:
            x = bf16_value(rec[..., at].astype(np.uint32) | (rec[..., at + 1].astype(np.uint32) << 8))
        else:
            b, E = rec[..., at].astype(np.int64), np.repeat(rec[..., exp_places(fmt, what)].astype(np.int64), 16, -1)
            if fmt == hma.HMA_KV_BFP8:
                x = np.ldexp(np.where(b > 127, -(b & 127), b).astype(np.float64), E - 133)
            else:
                x = np.ldexp(((b >> (4 * nib)) & 15).astype(np.float64) - 8, E - 129)
        got.append(np.moveaxis(x, 1, 2).reshape(-1, desc.num_kv_heads, 128))          # [pages][heads][16][128] -> [pages][16][heads][128]
    return got


class Paged:
    """A cache of random records and a permuted block table.  What no query may look at is poisoned: tokens behind the context and (for a
    window) hidden tokens hold NaN-like bytes, table entries of pages without a visible token are out of range."""

    def __init__(self, lens, hq, hkv, fmt, seed=0, spare=3, q_len=1, window=None, sinks=0, key_layout=0, layers=1, exps=(118, 131), extra_cols=0):
        import torch
        rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.fmt, self.q_len = np.asarray(lens, np.int32), hq, hkv, fmt, q_len
        npg = (np.maximum(self.lens, 0) + 15) // 16
        pages = int(npg.sum()) + spare
        self.desc = hma.make_desc(layers, hq, hkv, pages, fmt, key_layout=key_layout)
        ids = rng.permutation(pages).astype(np.int32)
        self.table = np.full((len(lens), max(int(npg.max()), 1) + extra_cols), -5, np.int32)
        o = 0
        for b, n in enumerate(npg):
            self.table[b, :n] = ids[o:o + n]
            o += n
        self.raw = []
        for _ in range(layers):
            layer = rng.integers(0, 256, hma.hma_cache_layer_bytes(self.desc), dtype=np.uint8)
            rec = records(layer, self.desc)
            if fmt == hma.HMA_KV_BF16:
                rec.view(np.uint16)[...] = bf16_round(rng.standard_normal(rec.view(np.uint16).shape).astype(np.float32))
            else:
                for what in (0, 1):
                    at = exp_places(fmt, what).reshape(-1)
                    rec[..., at] = rng.integers(*exps, rec[..., at].shape, dtype=np.uint8)
            self.raw.append(layer)
        self.clean = [r.copy() for r in self.raw]
        live = self.table.copy()
        for b, T in enumerate(self.lens):
            seen = np.zeros(int(npg[b]) * 16, bool)
            for i in range(q_len):
                end = max(0, int(T) - (q_len - 1 - i))
                t = np.arange(end)
                seen[:end] |= (t >= end - window) | (t < sinks) if window else True
            for p in range(int(npg[b])):
                if not seen[16 * p:16 * p + 16].any():
                    live[b, p] = -9 if p % 2 else 2 ** 30
                for t in np.flatnonzero(~seen[16 * p:16 * p + 16]):
                    for layer in self.raw:
                        r = records(layer, self.desc)[self.table[b, p]]
                        for what in (0, 1):
                            at, nib = places(fmt, what)
                            r[:, at[t]] = 255
                            if fmt == hma.HMA_KV_BF16:
                                r[:, at[t] + 1] = 255
                            else:
                                r[:, exp_places(fmt, what)[t]] = 255
        self.cache = hma.KVCache(self.desc, layers=[torch.from_numpy(r).cuda() for r in self.raw])
        self.tbl, self.ctx = torch.from_numpy(live).cuda(), torch.from_numpy(self.lens).cuda()
        shape = (len(lens), q_len, hq, 128)
        self.q = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16).cuda()
        self.scale = 1 / np.sqrt(128.0)

    def reference(self, layer=0, window=None, sinks=0, q=None, sequences=None):
        """float64 [batch][q_len][hq][128], and a bound on the kernel's fp32 error for each of its elements.

        Weights go to the tensor cores as FP16, relative to the largest one: a weight of 2^-14 or more is off by at most 2^-11 of
        itself, a smaller one (an FP16 subnormal, whose step is 2^-24) by at most 2^-25.  So numerator and denominator are each off by
        at most 2^-11 of the mean of |v| under the weights, plus 2^-25 for every token, times its |v| in the numerator and times the output in the denominator.  A score is a sum of 128 products of codes (up to 15 beside a value of up to 8, the offset) and
        queries, in 8 MMAs and 8 fp32 additions: at most 2^-19 of the sum of the products' magnitudes, which changes a weight by the same
        factor, twice (numerator and denominator)."""
        q = self.q if q is None else q
        q = q.double().cpu().numpy().reshape(len(self.lens), -1, self.hq, 128)
        if self.desc.key_layout:
            c = np.arange(128)
            q = q[..., (c >> 1) + 64 * (c & 1)]
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        G = self.hq // self.hkv
        for b in range(len(self.lens)) if sequences is None else sequences:
            T = int(self.lens[b])
            if T <= 0:
                continue
            k, v = read(self.clean[layer], self.desc, self.table[b, :(T + 15) // 16])
            for i in range(q.shape[1]):
                end = T - (q.shape[1] - 1 - i)
                if end <= 0:
                    continue
                t = np.arange(end)
                if window:
                    t = t[(t >= end - window) | (t < sinks)]
                for h in range(self.hkv):
                    qq, kk, vv = q[b, i, h * G:(h + 1) * G], k[t, h], v[t, h]
                    s = qq @ kk.T * self.scale
                    w = np.exp(s - s.max(1, keepdims=True))
                    w /= w.sum(1, keepdims=True)
                    out[b, i, h * G:(h + 1) * G] = w @ vv
                    # a step is at most the block's largest value unless all its codes are 8 (values zero): then nothing is off
                    size = np.abs(kk) if self.fmt != hma.HMA_KV_BFP4 else np.repeat(np.abs(kk).reshape(len(t), 8, 16).max(2), 16, 1) * 15
                    slip = 2.0 ** -19 * (np.abs(qq) @ size.T * self.scale).max(1, keepdims=True)
                    tol[b, i, h * G:(h + 1) * G] = (2.0 ** -10 + 2 * slip) * (w @ np.abs(vv)) + 2.0 ** -25 * (np.abs(vv).sum(0) + len(t) * np.abs(out[b, i, h * G:(h + 1) * G])) + 1e-30
        return out, tol

    def check(self, out32, out16, ref, tol):
        import torch
        got = out32.double().cpu().numpy().reshape(ref.shape)
        over = np.abs(got - ref) - tol
        assert np.isfinite(got).all() and (over <= 0).all(), (over.max(), np.unravel_index(over.argmax(), over.shape))
        assert (got[tol == 0] == 0).all()                          # rows that see nothing are zeros
        assert torch.equal(out16, out32.to(torch.bfloat16))        # the BF16 output is the FP32 one, rounded
        assert hma.hma_error_flags(self.cache) == 0
