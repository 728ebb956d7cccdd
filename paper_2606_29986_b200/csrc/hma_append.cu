// New tokens' K and V rows into the paged cache at given slots, and the same with the RMS norm of every query and key head
// and the rotation in front (hma_kv_append, hma_qk_norm_rope).
//
//   norm    y = x * rsqrt(mean(x^2) + eps) * w over the 128 channels of a head, sums in fp32
//   rotate  (a, b) -> (a cos - b sin, b cos + a sin) for every pair of the first rotary_dim channels
//   encode  E = the block's largest FP32 exponent field; codes = x * 2^(133 - E) (BFP8) or 2^(129 - E) (4-bit) rounded to nearest-even,
//           saturated at 127 / 7.  The scaling is a power of two, hence exact; FP32 subnormals encode as zero.
//
// Bound by HBM on long inputs (each row is read once and written once) and by latency on a decode batch, so everything is
// one launch.  A half-warp holds a row: 8 channels per lane, 16-byte loads, the norm's sum is four shuffles, a 16-channel
// block is two neighbouring lanes.  Two kinds of CTA share the grid:
//   * row CTAs write query (and, without a cache, key) rows.  A half-warp does up to 8 heads of one token, so that the
//     rotation's cosines and sines (512 B a token, against 256 B a row) are loaded once for all of them.
//   * cache CTAs take K or V of a kv head for a window of 16 tokens.  Inside a record the bytes of one token are
//     scattered (V of a BFP8 cache: single bytes), so 16 tokens that fill a whole page are put together in shared memory
//     and leave as whole words; other tokens (decode batches, ragged ends) store their bytes directly.  A page is
//     done by the CTA in whose window it starts.  A key's position and table row are read again for every head (a prompt of 8192
//     tokens, 64 + 8 heads, into a cache: 73 - 76 us; 50 at the copy rate).  Short inputs give a CTA one such part (two rows a half-warp, latency);
//     long ones give every warp a part of its own, with all of its rows in flight and no CTA barrier.
#include <cuda_bf16.h>

#include "hma_common.cuh"

namespace hma {

constexpr int kRowThreads = 128;                 // 8 half-warps
constexpr int kRowGroups = kRowThreads / 16;
// bytes of a staged row: 128 codes, 64 bytes of code pairs or 256 B of BF16, padded by 16 against bank conflicts
__host__ __device__ constexpr int stage_stride(int fmt) { return fmt == HMA_KV_BF16 ? 272 : fmt == HMA_KV_BFP8 ? 144 : 80; }
constexpr int kFmtNone = -1;
constexpr int kNoPage = -100;
constexpr int kManyRows = 4, kManyHeads = 8;     // rows a half-warp has in flight, and does in all, when there are many
constexpr int64_t kManyParts = 148 * 8;          // parts that the GPU holds at once, a CTA each
constexpr int64_t kFewRows = 148 * 5 * kRowGroups;    // half-warps that the GPU holds at once: until then one head each, then kManyRows, then kManyHeads
constexpr int64_t kMaxRowTokens = 1 << 24;

struct RowArgs {
    const uint8_t *k, *v;                        // K and V rows of token 0, head 0 (bytes; token strides in elements)
    int64_t k_stride, v_stride;
    const uint8_t *q;                            // query rows (hma_qk_norm_rope), token stride k_stride
    const uint8_t *q_weight, *k_weight;
    float eps;
    const float *rope;
    int64_t rope_rows;
    int half;                                    // rotary_dim / 2, 0: no rotation
    int interleaved;
    const int32_t *positions;
    uint16_t *q_out, *k_out;
    int64_t n_tokens;
    int hq, hkv;
    int row_heads;                               // heads a token has in the row part: hq, or hq + hkv when the keys are done there
    uint32_t cache_ctas;                         // the first CTAs of the grid; then those of the row part
    int unit_heads;                              // heads that a half-warp of the row part does
    uint32_t q_units, units_per_token;           // the first q_units of a token do its queries
    const int64_t *slots;
    uint8_t *layer;
    int64_t num_slots;
    int key_layout;
    uint32_t *flags;
};

// ---------------------------------------------------------------- one row in a half-warp
template <bool kF32>
__device__ __forceinline__ void load_row(const uint8_t *p, int lane16, float (&x)[8])
{
    if (kF32) {
        const float4 a = reinterpret_cast<const float4 *>(p)[2 * lane16], b = reinterpret_cast<const float4 *>(p)[2 * lane16 + 1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 v = reinterpret_cast<const uint4 *>(p)[lane16];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint4 pack_row(const float (&x)[8])
{
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ void norm_row(float (&x)[8], const float (&w)[8], float eps)
{
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, d);
    const float r = rsqrtf(fmaf(ss, 1.f / kHeadDim, eps));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
}
// This lane's cosines and sines for one position: half-split pairs (i, i + half) need 8 of each, neighbouring pairs 4.
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ void load_turn(const RowArgs &a, int64_t pos, int lane16, Turn &t)
{
    const int ch = 8 * lane16;
    const float *row = a.rope + pos * 2 * a.half;
#pragma unroll
    for (int i = 0; i < 8; ++i) { t.c[i] = 1.f; t.s[i] = 0.f; }
    if (ch >= 2 * a.half) return;
    if (a.interleaved) {
        const float4 c = *reinterpret_cast<const float4 *>(row + ch / 2), s = *reinterpret_cast<const float4 *>(row + a.half + ch / 2);
        t.c[0] = c.x; t.c[1] = c.y; t.c[2] = c.z; t.c[3] = c.w;
        t.s[0] = s.x; t.s[1] = s.y; t.s[2] = s.z; t.s[3] = s.w;
    } else {
        const int f = ch < a.half ? ch : ch - a.half;
        const float sign = ch < a.half ? -1.f : 1.f;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float4 c = *reinterpret_cast<const float4 *>(row + f + 4 * q), s = *reinterpret_cast<const float4 *>(row + a.half + f + 4 * q);
            t.c[4 * q] = c.x; t.c[4 * q + 1] = c.y; t.c[4 * q + 2] = c.z; t.c[4 * q + 3] = c.w;
            t.s[4 * q] = sign * s.x; t.s[4 * q + 1] = sign * s.y; t.s[4 * q + 2] = sign * s.z; t.s[4 * q + 3] = sign * s.w;
        }
    }
}
__device__ __forceinline__ void rotate_row(const RowArgs &a, int lane16, const Turn &t, float (&x)[8])
{
    if (a.interleaved) {
        if (8 * lane16 < 2 * a.half)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float u = x[2 * i], v = x[2 * i + 1];
                x[2 * i] = u * t.c[i] - v * t.s[i];
                x[2 * i + 1] = v * t.c[i] + u * t.s[i];
            }
    } else {
        const int step = a.half / 8, ch = 8 * lane16;
        const int mate = ch < a.half ? lane16 + step : ch < 2 * a.half ? lane16 - step : lane16;
        const bool turned = ch < 2 * a.half;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float o = __shfl_sync(0xFFFFFFFFu, x[i], mate, 16);
            if (turned) x[i] = x[i] * t.c[i] + o * t.s[i];          // an unturned channel passes as it is, infinities too
        }
    }
}
// query order -> cached order of a key whose cache keeps rotary pairs side by side (channel c <- (c >> 1) + 64 * (c & 1))
__device__ __forceinline__ void interleave_row(int lane16, float (&x)[8])
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int src = (lane16 >> 1) + 8 * (i & 1);
        const float lo = __shfl_sync(0xFFFFFFFFu, x[i >> 1], src, 16), hi = __shfl_sync(0xFFFFFFFFu, x[4 + (i >> 1)], src, 16);
        y[i] = (lane16 & 1) ? hi : lo;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i];
}
// A row as the cache holds it: BF16 values (w[0..3]), or one code a byte (w[0], w[1]) and the block's exponent byte.
struct Coded { uint32_t w[4], E; };
constexpr uint32_t kPlainLow = 30, kPlainHigh = 254;     // block exponents that need no care: subnormals vanish, the factor is an FP32 number
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// Four codes, a byte each, as the rounding left them: magnitudes 0 .. 128 with the signs in `sign`, or 8 + (-8 .. 8): saturated.
template <int kFmt>
__device__ __forceinline__ uint32_t saturate4(uint32_t m, uint32_t sign)
{
    if (kFmt == HMA_KV_BFP8) return (m - ((m >> 7) & 0x01010101u)) | (sign & 0x80808080u);      // 128 -> 127
    m -= (m >> 4) & 0x01010101u;                  // 16 (+8) -> 15
    return m | (~((m + 0x0F0F0F0Fu) >> 4) & 0x01010101u);      // 0 (-8) -> 1
}
// From FP32.  x * 2^(133 - E) (4-bit: 2^(129 - E)), a power of two, so exact; adding 2^23 (1.5 * 2^23 + 8) rounds it to an integer,
// halves to even, in the sum's low bits.
template <int kFmt>
__device__ __forceinline__ Coded encode_f32(const float (&x)[8], bool &bad)
{
    Coded r = {};
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_nan(top, fabsf(x[i]));
    top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    uint32_t E = __float_as_uint(top) >> 23;
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = x[i];
    if (__any_sync(0xFFFFFFFFu, E < kPlainLow || E > kPlainHigh)) {
        // rare: NaN or Inf (they count as zero), or a block so small that FP32 subnormals, which encode as zero, would scale
        // to something
        uint32_t e = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t f = (__float_as_uint(x[i]) >> 23) & 0xFFu;
            if (f == 0xFFu) bad = true;
            if (f == 0xFFu || f == 0u) c[i] = __uint_as_float(__float_as_uint(x[i]) & 0x80000000u);
            else e = max(e, f);
        }
        E = max(e, __shfl_xor_sync(0xFFFFFFFFu, e, 1));
    }
    r.E = E;
    const bool small = E < kPlainLow;             // then the factor is beyond FP32's largest and comes in two steps
    const float s1 = __uint_as_float((127u + (kFmt == HMA_KV_BFP8 ? 133u : 129u) - (small ? 20u : 0u) - E) << 23);
    if (__any_sync(0xFFFFFFFFu, small))
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] *= small ? 1048576.f : 1.f;
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        y[i] = __float_as_uint(kFmt == HMA_KV_BFP8 ? fmaf(fabsf(c[i]), s1, 8388608.f) : fmaf(c[i], s1, 12582920.f));
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint32_t m = __byte_perm(__byte_perm(y[4 * q], y[4 * q + 1], 0x0040), __byte_perm(y[4 * q + 2], y[4 * q + 3], 0x0040), 0x5410);
        uint32_t sign = 0;
        if (kFmt == HMA_KV_BFP8)
            sign = __byte_perm(__byte_perm(__float_as_uint(c[4 * q]), __float_as_uint(c[4 * q + 1]), 0x0073),
                               __byte_perm(__float_as_uint(c[4 * q + 2]), __float_as_uint(c[4 * q + 3]), 0x0073), 0x5410);
        r.w[q] = saturate4<kFmt>(m, sign);
    }
    return r;
}
// From BF16, two at a time: BF16 numbers between 128 and 256 are the integers, so one fused multiply-add in BF16 with 128 (136)
// rounds like the one above and leaves the code in the low byte; the largest magnitude is an integer maximum of the bits.
template <int kFmt>
__device__ __forceinline__ Coded encode_bf16(const uint4 &p, bool &bad)
{
    Coded r = {};
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
    if constexpr (kFmt == HMA_KV_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = w[i];
    } else {
        uint32_t mag[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) mag[i] = w[i] & 0x7FFF7FFFu;
        uint32_t top = __vmaxu2(__vmaxu2(mag[0], mag[1]), __vmaxu2(mag[2], mag[3]));
        top = __vmaxu2(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        const uint32_t E = max(top & 0xFFFFu, top >> 16) >> 7;
        if (__any_sync(0xFFFFFFFFu, E < kPlainLow || E > kPlainHigh)) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
            return encode_f32<kFmt>(x, bad);
        }
        r.E = E;
        const uint32_t s1 = ((127u + (kFmt == HMA_KV_BFP8 ? 133u : 129u) - E) << 7) * 0x00010001u;
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = kFmt == HMA_KV_BFP8 ? fma_bf16x2(mag[i], s1, 0x43004300u) : fma_bf16x2(w[i], s1, 0x43084308u);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (kFmt == HMA_KV_BFP8) r.w[q] = saturate4<kFmt>(__byte_perm(y[2 * q], y[2 * q + 1], 0x6420), __byte_perm(w[2 * q], w[2 * q + 1], 0x7531));
            else {                                // 8 + code, 0 .. 16, in the low bytes of the pairs: 1 .. 15
                const uint32_t lo = __vminu2(__vmaxu2(y[2 * q], 0x43014301u), 0x430F430Fu), hi = __vminu2(__vmaxu2(y[2 * q + 1], 0x43014301u), 0x430F430Fu);
                r.w[q] = __byte_perm(lo, hi, 0x6420);
            }
        }
    }
    return r;
}

// ---------------------------------------------------------------- a token's row straight into its record
// `part` is the record's K or V part, tok the token's place in its page; `other` (4-bit V) is what the lane's neighbour sent.
template <int kFmt, bool kV>
__device__ __forceinline__ void store_token(uint8_t *part, int tok, int lane16, const Coded &r, uint32_t other)
{
    const int j = lane16 >> 1, up = lane16 & 1, g = tok & 7, t8 = tok >> 3;       // block, the lane's half of it, ..
    const uint32_t lo = r.w[0], hi = r.w[1];
    if constexpr (kFmt != HMA_KV_BF16)
        if (!up) part[kV ? (g >> 1) * 32 + j * 4 + (tok & 1) + 2 * t8 : g * 16 + t8 * 8 + j] = (uint8_t)r.E;
    if constexpr (kFmt == HMA_KV_BF16 && !kV) {
        uint8_t *d = part + (t8 + 2 * (j >> 1)) * 512 + (g * 4 + 2 * up) * 16 + (j & 1) * 8;
        *reinterpret_cast<uint2 *>(d) = make_uint2(r.w[0], r.w[1]);
        *reinterpret_cast<uint2 *>(d + 16) = make_uint2(r.w[2], r.w[3]);
    } else if constexpr (kFmt == HMA_KV_BF16) {
        uint16_t *d = reinterpret_cast<uint16_t *>(part + j * 512 + (g >> 1) * 16 + (t8 * 2 + up) * 4 + (tok & 1) * 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i * 32] = (uint16_t)(r.w[i >> 1] >> (16 * (i & 1)));
    } else if constexpr (kFmt == HMA_KV_BFP8 && !kV) {
        uint8_t *d = part + 128 + (t8 + 2 * (j >> 2)) * 512 + (g * 4 + 2 * up) * 16 + (j & 3) * 4;
        *reinterpret_cast<uint32_t *>(d) = lo;
        *reinterpret_cast<uint32_t *>(d + 16) = hi;
    } else if constexpr (kFmt == HMA_KV_BFP8) {
        uint8_t *d = part + 128 + (j >> 1) * 512 + (g >> 1) * 16 + ((j & 1) * 2 + up) * 4 + (tok & 1) + 2 * t8;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i * 64] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
    } else if constexpr (!kV) {
        // 4-bit: a byte holds two codes of one token, so no other token's bits are touched
        uint8_t *d = part + 128 + (j >> 2) * 512 + (g * 4 + 2 * up) * 16 + (j & 3) * 4 + t8;
        d[0] = (uint8_t)((lo & 0xFFu) | ((lo >> 12) & 0xF0u));                 // channels 4t, 4t + 2
        d[2] = (uint8_t)(((lo >> 8) & 0xFFu) | ((lo >> 20) & 0xF0u));          // channels 4t + 1, 4t + 3
        d[16] = (uint8_t)((hi & 0xFFu) | ((hi >> 12) & 0xF0u));
        d[18] = (uint8_t)(((hi >> 8) & 0xFFu) | ((hi >> 20) & 0xF0u));
    } else {
        // channels c and c + 8 of the block share a byte: the lower lane stores c = 0..3, the upper one c = 4..7
        const uint32_t b = up ? other | (hi << 4) : lo | (other << 4);
        uint8_t *d = part + 128 + (j >> 2) * 512 + (16 * up + (g >> 1)) * 16 + (j & 3) * 4 + 2 * (tok & 1) + t8;
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i * 64] = (uint8_t)(b >> (8 * i));
    }
}

// ---------------------------------------------------------------- a whole page from its staged rows
// Staged row of a token: BF16 values, BFP8 codes a byte each, or 4-bit codes in the bytes that the record holds (K: bytes
// (4t, 4t + 2) and (4t + 1, 4t + 3) of every four channels; V: byte c of a block has its channels c and c + 8).
template <int kFmt, bool kV>
__device__ __forceinline__ void stage_row(uint8_t *d, int lane16, const Coded &r, uint32_t other)
{
    if constexpr (kFmt == HMA_KV_BF16) reinterpret_cast<uint4 *>(d)[lane16] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    else if constexpr (kFmt == HMA_KV_BFP8) reinterpret_cast<uint2 *>(d)[lane16] = make_uint2(r.w[0], r.w[1]);
    else if constexpr (kV) reinterpret_cast<uint32_t *>(d)[lane16] = (lane16 & 1) ? other | (r.w[1] << 4) : r.w[0] | (other << 4);
    else {
        const uint32_t p = r.w[0] | (r.w[0] >> 12), q = r.w[1] | (r.w[1] >> 12);      // low bytes: codes (0, 2) and (1, 3)
        reinterpret_cast<uint32_t *>(d)[lane16] = __byte_perm(p, q, 0x5410);
    }
}
// Written by kThreads threads, of which this is number `id`; exps[t] are token t's exponents.
template <int kFmt, bool kV, int kThreads>
__device__ __forceinline__ void store_page(uint8_t *part, const uint8_t (*rows)[stage_stride(kFmt)], const uint8_t (*exps)[8], int id)
{
    if (kFmt != HMA_KV_BF16 && id >= kThreads - 32) {            // exponent bytes, one word a thread of the last warp
        const int w = id - (kThreads - 32);
        uint32_t v;
        if (!kV) v = *reinterpret_cast<const uint32_t *>(&exps[(w >> 2) + 8 * ((w >> 1) & 1)][4 * (w & 1)]);
        else {
            const int t2 = 2 * (w >> 3), j = w & 7;
            v = exps[t2][j] | (exps[t2 + 1][j] << 8) | (exps[t2 + 8][j] << 16) | ((uint32_t)exps[t2 + 9][j] << 24);
        }
        reinterpret_cast<uint32_t *>(part)[w] = v;
    }
    if constexpr (kV && kFmt != HMA_KV_BF16) {
        // four tokens (2t, 2t + 1, 2t + 8, 2t + 9) by four bytes of their rows: four words of the record, transposed in registers
        constexpr int kQuads = kFmt == HMA_KV_BFP8 ? 32 : 16;                // words of a staged row
#pragma unroll
        for (int q = id; q < 4 * kQuads; q += kThreads) {
            const int t = q & 3, x = q >> 2;
            // neighbouring threads take the same bytes of neighbouring blocks: their words are neighbours in the record
            const int word = (x & 3) * 2 + (x >> 2 & 1) + 8 * (x >> 3);
            const uint32_t w0 = *reinterpret_cast<const uint32_t *>(&rows[2 * t][4 * word]), w1 = *reinterpret_cast<const uint32_t *>(&rows[2 * t + 1][4 * word]);
            const uint32_t w8 = *reinterpret_cast<const uint32_t *>(&rows[2 * t + 8][4 * word]), w9 = *reinterpret_cast<const uint32_t *>(&rows[2 * t + 9][4 * word]);
            // BFP8 words hold the tokens in the order 2t, 2t + 1, 2t + 8, 2t + 9; 4-bit ones 2t, 2t + 8, 2t + 1, 2t + 9
            const uint32_t b = kFmt == HMA_KV_BFP8 ? w1 : w8, c = kFmt == HMA_KV_BFP8 ? w8 : w1;
            const uint32_t a01 = __byte_perm(w0, b, 0x5140), b01 = __byte_perm(w0, b, 0x7362), a23 = __byte_perm(c, w9, 0x5140), b23 = __byte_perm(c, w9, 0x7362);
            const uint32_t o[4] = {__byte_perm(a01, a23, 0x5410), __byte_perm(a01, a23, 0x7632), __byte_perm(b01, b23, 0x5410), __byte_perm(b01, b23, 0x7632)};
            uint8_t *d;
            if (kFmt == HMA_KV_BFP8) {
                const int j = word >> 2, half = word >> 1 & 1, g = 4 * (word & 1);           // channels 16j + 8 * half + g ..
                d = part + 128 + (j >> 1) * 512 + (g * 4 + t) * 16 + ((j & 1) * 2 + half) * 4;
            } else {
                const int j = word >> 1, g = 4 * (word & 1);
                d = part + 128 + (j >> 2) * 512 + (g * 4 + t) * 16 + (j & 3) * 4;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t *>(d + i * 64) = o[i];
        }
    } else {
        constexpr int kHead = kFmt == HMA_KV_BF16 ? 0 : 128;
        constexpr int kWords = (kFmt == HMA_KV_BFP8 ? 2048 : kFmt == HMA_KV_BF16 ? 4096 : 1024) / 16;
#pragma unroll
        for (int i = id; i < kWords; i += kThreads) {
            const int c = i >> 5, g = (i >> 2) & 7, t = i & 3;       // 512-byte piece, lane = 4 * g + t
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (kFmt == HMA_KV_BFP8) {
                    w[k] = *reinterpret_cast<const uint32_t *>(&rows[g + 8 * (c & 1)][16 * (4 * (c >> 1) + k) + 4 * t]);
                } else if constexpr (kFmt == HMA_KV_BF16 && !kV) {
                    w[k] = *reinterpret_cast<const uint32_t *>(&rows[g + 8 * (c & 1)][2 * (16 * (2 * (c >> 1) + (k >> 1)) + 4 * t + 2 * (k & 1))]);
                } else if constexpr (kFmt == HMA_KV_BF16) {
                    const int ch = 16 * c + 8 * (k & 1) + g, tok = 2 * t + 8 * (k >> 1);
                    w[k] = *reinterpret_cast<const uint16_t *>(&rows[tok][2 * ch]) | ((uint32_t)*reinterpret_cast<const uint16_t *>(&rows[tok + 1][2 * ch]) << 16);
                } else {
                    const int at = 8 * (4 * c + k) + 2 * t;
                    w[k] = __byte_perm(*reinterpret_cast<const uint16_t *>(&rows[g][at]), *reinterpret_cast<const uint16_t *>(&rows[g + 8][at]), 0x5140);
                }
            }
            *reinterpret_cast<uint4 *>(part + kHead + 16 * i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// ---------------------------------------------------------------- the kernel
// A lane's 8 channels of a row as they are in memory.
template <bool kF32> struct Raw { uint4 v[kF32 ? 2 : 1]; };
template <bool kF32>
__device__ __forceinline__ Raw<kF32> fetch_row(const uint8_t *p, int lane16)
{
    Raw<kF32> r;
#pragma unroll
    for (int i = 0; i < (kF32 ? 2 : 1); ++i) r.v[i] = reinterpret_cast<const uint4 *>(p)[(kF32 ? 2 : 1) * lane16 + i];
    return r;
}
template <bool kF32>
__device__ __forceinline__ void widen(const Raw<kF32> &r, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kF32) {
            const uint4 &a = r.v[i >> 1];
            x[2 * i] = __uint_as_float((i & 1) ? a.z : a.x);
            x[2 * i + 1] = __uint_as_float((i & 1) ? a.w : a.y);
        } else {
            const uint32_t w = i == 0 ? r.v[0].x : i == 1 ? r.v[0].y : i == 2 ? r.v[0].z : r.v[0].w;
            x[2 * i] = __uint_as_float(w << 16);
            x[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
        }
    }
}
__device__ __forceinline__ int64_t position_of(const RowArgs &a, int64_t tok, int lane16)
{
    const int64_t p = a.positions[tok];
    if (p >= 0 && p < a.rope_rows) return p;
    if (lane16 == 0) atomicOr(a.flags, HMA_FLAG_BAD_POSITION);
    return 0;                                     // the table's first row: in bounds, and flagged
}

// Two FP32 operations an instruction (packed pairs in 64-bit registers).
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 pair(float lo, float hi) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ void split(F2 a, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

// A half-warp's share of the row part: `count` heads of one token and one kind.
struct RowUnit {
    const uint8_t *src;                          // its first row, and where that goes
    uint16_t *dst;
    const uint8_t *weight;
    int count;                                   // 0: no work, but the half-warp stays for its warp's shuffles
    int64_t tok;
};
// Rotation of all 128 channels as half-split pairs (the usual one): a lane holds channels 4l .. 4l + 3 and 64 + 4l .. 64 + 4l + 3, so that
// both members of its pairs are its own and nothing is exchanged.  Per row and lane: 4 packed operations for the sum of
// squares, 8 for the scaling, 8 for the rotation.  kRows rows are worked on while the next kRows are on their way.
template <bool kF32, int kRows>
__device__ __forceinline__ void rows_split64(const RowArgs &a, const RowUnit &u, int lane16)
{
    constexpr int kElem = kF32 ? 4 : 2;
    struct Half { uint32_t v[kF32 ? 4 : 2]; };
    auto load4 = [&](const uint8_t *p, int part) {
        Half x;
        if constexpr (kF32) {
            const uint4 v = reinterpret_cast<const uint4 *>(p)[16 * part + lane16];
            x.v[0] = v.x; x.v[1] = v.y; x.v[2] = v.z; x.v[3] = v.w;
        } else {
            const uint2 v = reinterpret_cast<const uint2 *>(p)[16 * part + lane16];
            x.v[0] = v.x; x.v[1] = v.y;
        }
        return x;
    };
    auto wide = [&](const Half &x, int i) {
        if constexpr (kF32) return pair(__uint_as_float(x.v[2 * i]), __uint_as_float(x.v[2 * i + 1]));
        else return pair(__uint_as_float(x.v[i] << 16), __uint_as_float(x.v[i] & 0xFFFF0000u));
    };
    Half x[kRows][2] = {};
    auto fetch = [&](int h) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (h + r < u.count)
#pragma unroll
                for (int p = 0; p < 2; ++p) x[r][p] = load4(u.src + (int64_t)(h + r) * kHeadDim * kElem, p);
    };
    fetch(0);
    const float *row = a.rope + position_of(a, u.tok, lane16) * kHeadDim;
    const float4 cv = *reinterpret_cast<const float4 *>(row + 4 * lane16), sv = *reinterpret_cast<const float4 *>(row + 64 + 4 * lane16);
    const F2 c[2] = {pair(cv.x, cv.y), pair(cv.z, cv.w)}, s[2] = {pair(sv.x, sv.y), pair(sv.z, sv.w)}, ns[2] = {pair(-sv.x, -sv.y), pair(-sv.z, -sv.w)};
    F2 w[2][2];
    if (u.weight) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const Half f = load4(u.weight, p);
            w[p][0] = wide(f, 0);
            w[p][1] = wide(f, 1);
        }
    }
    for (int h = 0; h < a.unit_heads; h += kRows) {      // every half-warp makes the same number of steps: its warp's shuffles are in step
        F2 v[kRows][2][2];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int p = 0; p < 2; ++p) { v[r][p][0] = wide(x[r][p], 0); v[r][p][1] = wide(x[r][p], 1); }
        fetch(h + kRows);
        float ss[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            F2 q = mul2(v[r][0][0], v[r][0][0]);
            q = fma2(v[r][0][1], v[r][0][1], q); q = fma2(v[r][1][0], v[r][1][0], q); q = fma2(v[r][1][1], v[r][1][1], q);
            float s0, s1;
            split(q, s0, s1);
            ss[r] = s0 + s1;
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1)
#pragma unroll
            for (int r = 0; r < kRows; ++r) ss[r] += __shfl_xor_sync(0xFFFFFFFFu, ss[r], d);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (u.weight) {
                const float f = rsqrtf(fmaf(ss[r], 1.f / kHeadDim, a.eps));
                const F2 ff = pair(f, f);
#pragma unroll
                for (int p = 0; p < 2; ++p) { v[r][p][0] = mul2(mul2(v[r][p][0], ff), w[p][0]); v[r][p][1] = mul2(mul2(v[r][p][1], ff), w[p][1]); }
            }
            uint32_t out[2][2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const F2 lo = fma2(v[r][0][q], c[q], mul2(v[r][1][q], ns[q])), hi = fma2(v[r][1][q], c[q], mul2(v[r][0][q], s[q]));
                float u0, u1;
                split(lo, u0, u1);
                out[0][q] = pack_bf16(u0, u1);
                split(hi, u0, u1);
                out[1][q] = pack_bf16(u0, u1);
            }
            if (h + r < u.count) {
                uint2 *o = reinterpret_cast<uint2 *>(u.dst + (int64_t)(h + r) * kHeadDim);
                o[lane16] = make_uint2(out[0][0], out[0][1]);
                o[16 + lane16] = make_uint2(out[1][0], out[1][1]);
            }
        }
    }
}
// The same for any other rotation (a part of the channels, neighbouring pairs, none): 8 neighbouring channels a lane.
template <bool kF32, int kRows>
__device__ __forceinline__ void rows_any(const RowArgs &a, const RowUnit &u, int lane16)
{
    constexpr int kElem = kF32 ? 4 : 2;
    Raw<kF32> raw[kRows] = {};
    auto fetch = [&](int h) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (h + r < u.count) raw[r] = fetch_row<kF32>(u.src + (int64_t)(h + r) * kHeadDim * kElem, lane16);
    };
    fetch(0);
    Turn turn;
    if (a.half) load_turn(a, position_of(a, u.tok, lane16), lane16, turn);
    float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (u.weight) load_row<kF32>(u.weight, lane16, w);
    for (int h = 0; h < a.unit_heads; h += kRows) {
        float x[kRows][8];
#pragma unroll
        for (int r = 0; r < kRows; ++r) widen<kF32>(raw[r], x[r]);
        fetch(h + kRows);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[r][e];
            norm_row(y, w, a.eps);                // both half-warps of a warp run the same shuffles, whatever their heads are
            if (u.weight)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[r][e] = y[e];
            if (a.half) rotate_row(a, lane16, turn, x[r]);
            if (h + r < u.count) reinterpret_cast<uint4 *>(u.dst + (int64_t)(h + r) * kHeadDim)[lane16] = pack_row(x[r]);
        }
    }
}

// kNorm: hma_qk_norm_rope (else hma_kv_append: no row CTAs).  kFmt: format of the cache, kFmtNone without one.  The cache CTAs
// come first in the grid: theirs is the longest chain of loads.  kGroups: half-warps that share a part, 8 (the CTA) or 2 (a warp).
template <bool kF32, int kFmt, bool kNorm, int kRows, int kGroups>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const RowArgs a)
{
    constexpr int kElem = kF32 ? 4 : 2;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
    if (kNorm && blockIdx.x >= a.cache_ctas) {
        const uint32_t unit = (blockIdx.x - a.cache_ctas) * kRowGroups + grp;
        const uint32_t t = unit / a.units_per_token, i = unit - t * a.units_per_token;
        const bool key = i >= a.q_units;
        const int h0 = (int)(key ? i - a.q_units : i) * a.unit_heads, heads = key ? a.hkv : a.hq;
        RowUnit u;
        u.tok = min((int64_t)t, a.n_tokens - 1);
        u.count = t < (uint32_t)a.n_tokens ? min(heads - h0, a.unit_heads) : 0;
        u.src = (key ? a.k : a.q) + (u.tok * a.k_stride + (int64_t)h0 * kHeadDim) * kElem;
        u.dst = key ? a.k_out + (u.tok * a.hkv + h0) * kHeadDim : a.q_out + (u.tok * a.hq + h0) * kHeadDim;
        u.weight = key ? a.k_weight : a.q_weight;
        if (a.half == 64 && !a.interleaved) rows_split64<kF32, kRows>(a, u, lane16);
        else rows_any<kF32, kRows>(a, u, lane16);
        return;
    }
    if constexpr (kFmt != kFmtNone) {
        constexpr int kParts = kRowGroups / kGroups, kOwn = kPageTokens / kGroups, kThreads = 16 * kGroups;
        __shared__ __align__(16) uint8_t rows[kParts][kPageTokens][stage_stride(kFmt)];
        __shared__ __align__(4) uint8_t exps[kParts][kPageTokens][8];
        const int mine = grp / kGroups, g0 = grp % kGroups;                       // the thread's part of the CTA's, its half-warp there
        const uint32_t per_window = (uint32_t)(2 * a.hkv + kParts - 1) / kParts;  // CTAs that share a window
        const int64_t base = (int64_t)(blockIdx.x / per_window) * kPageTokens;
        const int hw = (int)(blockIdx.x % per_window) * kParts + mine, head = hw >> 1;      // head * 2 + (0: K, 1: V)
        const bool is_v = hw & 1, idle = hw >= 2 * a.hkv;
        const int64_t n = a.n_tokens;
        const int64_t stride = (is_v ? a.v_stride : a.k_stride) * kElem;
        const uint8_t *const src = (is_v ? a.v : a.k) + (int64_t)(idle ? 0 : head) * kHeadDim * kElem;
        // the window's rows are requested at once; whether they are wanted shows when the slots are here
        const uint8_t *const src0 = src + (base + g0) * stride;
        const bool full = base + kPageTokens <= n;
        Raw<kF32> own[kOwn];
#pragma unroll
        for (int r = 0; r < kOwn; ++r) own[r] = fetch_row<kF32>(full ? src0 + r * kGroups * stride : src + min(base + r * kGroups + g0, n - 1) * stride, lane16);
        // whole pages: runs of 16 consecutive slots from a multiple of 16.  Every warp looks for them in the slots of tokens base - 15
        // .. base + 30, bit i of a mask for token base - 15 + i.
        const int lane = threadIdx.x & 31;
        auto slot_at = [&](int64_t i) { return i >= 0 && i < n ? a.slots[i] : -1; };
        const int64_t lo = slot_at(base - 15 + lane), hi = lane < 14 ? slot_at(base + 17 + lane) : -1;
        const int64_t hi0 = __shfl_sync(0xFFFFFFFFu, hi, 0), lo_up = __shfl_down_sync(0xFFFFFFFFu, lo, 1), hi_up = __shfl_down_sync(0xFFFFFFFFu, hi, 1);
        uint64_t run = __ballot_sync(0xFFFFFFFFu, lo >= 0 && (uint64_t)(lane == 31 ? hi0 : lo_up) == (uint64_t)lo + 1);      // the next token's slot follows
        run |= (uint64_t)__ballot_sync(0xFFFFFFFFu, hi >= 0 && (uint64_t)hi_up == (uint64_t)hi + 1) << 32;
        run &= run >> 1; run &= run >> 2; run &= run >> 4; run &= run >> 7;                               // 15 times in a row
        const uint32_t starts = (uint32_t)run & __ballot_sync(0xFFFFFFFFu, lo >= 0 && lo <= a.num_slots - kPageTokens /* (no sum: any number may stand there) */ && lo % kPageTokens == 0) & 0x7FFFFFFFu;
        // whole pages do not overlap: at most one starts before the window and reaches into it, and one starts inside
        const int before_end = (starts & 0x7FFFu) ? 31 - __clz(starts & 0x7FFFu) - 15 + kPageTokens : 0;      // tokens below are another CTA's
        const int page_at = (starts >> 15) ? __ffs(starts >> 15) - 1 : kNoPage;
        if (kParts > 1 && idle) return;           // a whole warp; there is no CTA barrier then
        constexpr int64_t kHalf = record_bytes(kFmt) / 2;
        const int64_t page_bytes = (int64_t)a.hkv * 2 * kHalf;
        uint8_t *const first = a.layer + (int64_t)hw * kHalf;                     // this part of page 0
        float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (kNorm && !is_v && a.k_weight) load_row<kF32>(a.k_weight, lane16, w);
        bool bad = false;
        // one token's row: `staged` its row in the page that is put together here (or -1), `place` whether it is stored by itself at slot s
        auto one = [&](const Raw<kF32> &raw, int i, int staged, bool place, int64_t s, bool sure) {
            const bool key_row = kNorm && !is_v && a.k_out != nullptr && i < kPageTokens && base + i < n;      // the window's own keys, cached or not
            if (!sure && !__any_sync(0xFFFFFFFFu, staged >= 0 || place || key_row)) return;    // a half-warp without work goes along with the other one
            bool odd = false;
            Coded r;
            if (kF32 || (kNorm && !is_v) || (!is_v && a.key_layout == HMA_KEYS_INTERLEAVED)) {
                float x[8];
                widen<kF32>(raw, x);
                if (kNorm && !is_v) {
                    if (a.k_weight) norm_row(x, w, a.eps);
                    if (a.half) {
                        Turn turn;
                        load_turn(a, position_of(a, min(base + i, n - 1), lane16), lane16, turn);
                        rotate_row(a, lane16, turn, x);
                    }
                    // the key is what k_out says: rounded to BF16 once, and that value is cached
                    const uint4 p = pack_row(x);
                    const uint32_t b[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(b[k] << 16); x[2 * k + 1] = __uint_as_float(b[k] & 0xFFFF0000u); }
                    if (key_row) reinterpret_cast<uint4 *>(a.k_out + ((base + i) * a.hkv + head) * kHeadDim)[lane16] = p;
                }
                if (!is_v && a.key_layout == HMA_KEYS_INTERLEAVED) interleave_row(lane16, x);
                if constexpr (kFmt == HMA_KV_BF16) r = encode_bf16<kFmt>(pack_row(x), odd);
                else if (kF32 && (is_v || !kNorm)) r = encode_f32<kFmt>(x, odd);
                else r = encode_bf16<kFmt>(pack_row(x), odd);
            } else {
                r = encode_bf16<kFmt>(raw.v[0], odd);
            }
            bad |= odd && (sure || staged >= 0 || place);
            const uint32_t other = kFmt == HMA_KV_BFP4 ? __shfl_xor_sync(0xFFFFFFFFu, (lane16 & 1) ? r.w[0] : r.w[1], 1) : 0u;
            if (sure || staged >= 0) {
                if (is_v) stage_row<kFmt, true>(rows[mine][staged], lane16, r, other);
                else stage_row<kFmt, false>(rows[mine][staged], lane16, r, other);
                if (kFmt != HMA_KV_BF16 && !(lane16 & 1)) exps[mine][staged][lane16 >> 1] = (uint8_t)r.E;
            } else if (place) {
                uint8_t *record = first + s / kPageTokens * page_bytes;
                if (is_v) store_token<kFmt, true>(record, (int)(s % kPageTokens), lane16, r, other);
                else store_token<kFmt, false>(record, (int)(s % kPageTokens), lane16, r, other);
            }
        };
        if (page_at == 0) {                       // the window is one page
#pragma unroll
            for (int r = 0; r < kOwn; ++r) one(own[r], r * kGroups + g0, r * kGroups + g0, false, 0, true);
        } else {
            // (read again, from the first-level cache: a second unrolled copy of the loop would cost more in instruction fetches)
#pragma unroll 1
            for (int r = 0; r < kOwn; ++r) {
                const int i = r * kGroups + g0;
                const int64_t s = __shfl_sync(0xFFFFFFFFu, lo, 15 + i);
                const int staged = page_at != kNoPage && i >= page_at ? i - page_at : -1;
                const bool single = staged < 0 && i >= before_end && s != -1;
                const bool place = single && s >= 0 && s < a.num_slots;
                if (single && !place && lane16 == 0) atomicOr(a.flags, HMA_FLAG_BAD_PAGE_INGEST);
                one(fetch_row<kF32>(src + min(base + i, n - 1) * stride, lane16), i, staged, place, s, false);
            }
            // the rest of a page that starts here and ends in the next window
#pragma unroll 1
            for (int i = kPageTokens + g0; i - g0 < page_at + kPageTokens; i += kGroups)
                one(fetch_row<kF32>(src + min(base + i, n - 1) * stride, lane16), i, i < page_at + kPageTokens ? i - page_at : -1, false, 0, false);
        }
        if (bad) atomicOr(a.flags, HMA_FLAG_BAD_VALUE_ENCODE);
        if (page_at == kNoPage) return;           // the same in every thread of the part
        const int64_t page = __shfl_sync(0xFFFFFFFFu, lo, 15 + page_at) / kPageTokens;
        if (kParts == 1) __syncthreads();
        else __syncwarp();
        const int id = threadIdx.x % kThreads;
        uint8_t *part = first + page * page_bytes;
        if (is_v) store_page<kFmt, true, kThreads>(part, rows[mine], exps[mine], id);
        else store_page<kFmt, false, kThreads>(part, rows[mine], exps[mine], id);
    }
}

template <bool kF32, int kFmt, bool kNorm>
static cudaError_t launch_rows(RowArgs &a, cudaStream_t s)
{
    // a part (K or V of one head, 16 tokens) for each CTA until the GPU is full of them, then for each warp
    const int64_t windows = kFmt == kFmtNone ? 0 : (a.n_tokens + kPageTokens - 1) / kPageTokens, parts = windows * 2 * a.hkv;
    const bool by_warp = parts > kManyParts;
    const int64_t cache_ctas = by_warp ? windows * ((2 * a.hkv + 3) / 4) : parts;
    a.cache_ctas = (uint32_t)cache_ctas;
    int64_t row_ctas = 0;
    bool few = true;
    if constexpr (kNorm) {
        const int64_t rows = a.n_tokens * a.row_heads;
        few = rows <= kFewRows;
        a.unit_heads = few ? 1 : rows <= kFewRows * kManyHeads ? kManyRows : kManyHeads;
        a.q_units = (uint32_t)((a.hq + a.unit_heads - 1) / a.unit_heads);
        a.units_per_token = a.q_units + (uint32_t)((a.row_heads - a.hq + a.unit_heads - 1) / a.unit_heads);
        row_ctas = (a.n_tokens * a.units_per_token + kRowGroups - 1) / kRowGroups;
    }
    constexpr int kLong = kNorm ? kManyRows : 1, kWarp = kFmt == kFmtNone ? 8 : 2;
    // (a part for each warp means more than kManyParts * 8 - 15 * kMaxKvHeads rows, hence never few of them: the norm has three variants, not four)
    static_assert(kManyParts * kPageTokens / 2 - (kPageTokens - 1) * kMaxKvHeads > kFewRows, "few rows are few parts");
    void (*kernel)(const RowArgs) = by_warp ? rows_kernel<kF32, kFmt, kNorm, kLong, kWarp> : few ? rows_kernel<kF32, kFmt, kNorm, 1, 8> : rows_kernel<kF32, kFmt, kNorm, kLong, 8>;
    return launch_after(kernel, dim3((unsigned)(row_ctas + cache_ctas)), kRowThreads, 0, s, a);
}
template <bool kNorm>
static cudaError_t launch_rows_any(RowArgs &a, bool f32, int fmt, cudaStream_t s)
{
    if (fmt == HMA_KV_BFP8) return f32 ? launch_rows<true, HMA_KV_BFP8, kNorm>(a, s) : launch_rows<false, HMA_KV_BFP8, kNorm>(a, s);
    if (fmt == HMA_KV_BFP4) return f32 ? launch_rows<true, HMA_KV_BFP4, kNorm>(a, s) : launch_rows<false, HMA_KV_BFP4, kNorm>(a, s);
    if (fmt == HMA_KV_BF16) return f32 ? launch_rows<true, HMA_KV_BF16, kNorm>(a, s) : launch_rows<false, HMA_KV_BF16, kNorm>(a, s);
    if constexpr (kNorm) return f32 ? launch_rows<true, kFmtNone, kNorm>(a, s) : launch_rows<false, kFmtNone, kNorm>(a, s);
    return cudaErrorInvalidValue;
}
static void set_cache(RowArgs &a, const hma_cache *c, int layer, const int64_t *slots)
{
    a.hkv = c->desc.num_kv_heads;
    a.slots = slots;
    a.layer = (uint8_t *)c->layers[layer];
    a.num_slots = c->desc.num_pages * kPageTokens;
    a.key_layout = c->desc.key_layout;
    a.flags = c->flags;
}

}  // namespace hma

extern "C" hma_status_t hma_kv_append(hma_cache_t *cache, int32_t layer, const void *k, const void *v, int32_t in_dtype,
                                      int64_t k_token_stride, int64_t v_token_stride, const int64_t *slots, int64_t n_tokens,
                                      void *stream)
{
    if (!cache || layer < 0 || layer >= cache->desc.num_layers || n_tokens < 0) return HMA_ERR_INVALID_ARG;
    if (!hma::on_cache_device(cache)) return HMA_ERR_INVALID_ARG;
    if (in_dtype != HMA_OUT_BF16 && in_dtype != HMA_OUT_F32) return HMA_ERR_INVALID_ARG;
    const int64_t row = (int64_t)cache->desc.num_kv_heads * hma::kHeadDim;
    if (n_tokens <= 1) k_token_stride = v_token_stride = row;      // no second token: not looked at
    if (k_token_stride < row || v_token_stride < row) return HMA_ERR_INVALID_ARG;
    if (n_tokens > hma::kMaxRowTokens || k_token_stride > (1 << 30) || v_token_stride > (1 << 30)) return HMA_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens == 0) return HMA_OK;
    if (!k || !v || !slots) return HMA_ERR_INVALID_ARG;
    const int64_t elem = in_dtype == HMA_OUT_F32 ? 4 : 2;
    if (((uintptr_t)k & 15u) || ((uintptr_t)v & 15u) || (k_token_stride * elem & 15) || (v_token_stride * elem & 15)) return HMA_ERR_ALIGNMENT;
    hma::RowArgs a = {};
    a.k = (const uint8_t *)k; a.v = (const uint8_t *)v;
    a.k_stride = k_token_stride; a.v_stride = v_token_stride;
    a.n_tokens = n_tokens;
    hma::set_cache(a, cache, layer, slots);
    HMA_CUDA_OK(hma::launch_rows_any<false>(a, in_dtype == HMA_OUT_F32, cache->desc.format, (cudaStream_t)stream));
    hma::count_launch();
    return HMA_OK;
}

extern "C" hma_status_t hma_qk_norm_rope(hma_cache_t *cache, int32_t layer, const void *qkv, int32_t in_dtype, int64_t token_stride,
                                         int64_t n_tokens, const void *q_weight, const void *k_weight, float eps,
                                         const float *rope_table, int64_t rope_rows, int32_t rotary_dim, int32_t interleaved,
                                         const int32_t *positions, const int64_t *slots, void *q_out, void *k_out, void *stream)
{
    if (!cache || layer < 0 || layer >= cache->desc.num_layers || n_tokens < 0 || !(eps >= 0.f)) return HMA_ERR_INVALID_ARG;
    if (!hma::on_cache_device(cache)) return HMA_ERR_INVALID_ARG;
    if ((in_dtype != HMA_OUT_BF16 && in_dtype != HMA_OUT_F32) || (interleaved != 0 && interleaved != 1)) return HMA_ERR_INVALID_ARG;
    if (rotary_dim < 0 || rotary_dim > hma::kHeadDim || rotary_dim % 16) return HMA_ERR_UNSUPPORTED_SHAPE;
    const int hq = cache->desc.num_q_heads, hkv = cache->desc.num_kv_heads;
    const int64_t row = (int64_t)(hq + 2 * hkv) * hma::kHeadDim;
    if (n_tokens <= 1) token_stride = row;        // no second token: not looked at
    if (token_stride < row) return HMA_ERR_INVALID_ARG;
    if (n_tokens > hma::kMaxRowTokens || token_stride > (1 << 30)) return HMA_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens == 0) return HMA_OK;
    if (!qkv || !q_out || (!slots && !k_out) || (rotary_dim && (!rope_table || !positions || rope_rows < 1))) return HMA_ERR_INVALID_ARG;
    const int64_t elem = in_dtype == HMA_OUT_F32 ? 4 : 2;
    if (((uintptr_t)qkv & 15u) || (token_stride * elem & 15) || ((uintptr_t)q_weight & 15u) || ((uintptr_t)k_weight & 15u) ||
        ((uintptr_t)rope_table & 15u) || ((uintptr_t)q_out & 15u) || ((uintptr_t)k_out & 15u))
        return HMA_ERR_ALIGNMENT;
    hma::RowArgs a = {};
    a.q = (const uint8_t *)qkv;
    a.k = a.q + (int64_t)hq * hma::kHeadDim * elem;
    a.v = a.k + (int64_t)hkv * hma::kHeadDim * elem;
    a.k_stride = a.v_stride = token_stride;
    a.q_weight = (const uint8_t *)q_weight; a.k_weight = (const uint8_t *)k_weight;
    a.eps = eps;
    a.rope = rope_table; a.rope_rows = rope_rows; a.half = rotary_dim / 2; a.interleaved = interleaved; a.positions = positions;
    a.q_out = (uint16_t *)q_out; a.k_out = (uint16_t *)k_out;
    a.n_tokens = n_tokens;
    a.hq = hq;
    a.row_heads = slots ? hq : hq + hkv;
    hma::set_cache(a, cache, layer, slots);
    HMA_CUDA_OK(hma::launch_rows_any<true>(a, in_dtype == HMA_OUT_F32, slots ? cache->desc.format : hma::kFmtNone, (cudaStream_t)stream));
    hma::count_launch();
    return HMA_OK;
}
