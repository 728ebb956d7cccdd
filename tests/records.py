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
