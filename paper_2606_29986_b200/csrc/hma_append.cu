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
//   * row CTAs write query (and, without a cache, key) rows.  A half-warp does kRows heads of one token, so that the
//     rotation's cosines and sines (512 B a token, against 256 B a row) are loaded once for all of them.
//   * cache CTAs take one kv head of K or of V for a window of 16 tokens.  Inside a record the bytes of one token are
//     scattered (V of a BFP8 cache: single bytes), so 16 tokens that fill a whole page are put together in shared memory
//     and leave as 16-byte words; other tokens (decode batches, ragged ends) store their bytes directly.  A page is
//     done by the CTA in whose window it starts.
#include <cuda_bf16.h>

#include "hma_common.cuh"

namespace hma {

constexpr int kRowThreads = 128;                 // 8 half-warps
constexpr int kRowGroups = kRowThreads / 16;
constexpr int kStageStride = 272;                // bytes of a staged row: 128 codes or 256 B of BF16, padded by 16 against bank conflicts
constexpr int kFmtNone = -1;
constexpr int kNoPage = -100;
constexpr int kManyRows = 4;                     // heads a half-warp does when there are many rows
constexpr int64_t kFewRows = 148 * 16 * kRowGroups;   // rows that the GPU holds at once, one a half-warp: until then one head each
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
    int64_t row_ctas;
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
template <int kFmt>
__device__ __forceinline__ Coded encode_row(const float (&x)[8], bool &bad)
{
    Coded r = {};
    if constexpr (kFmt == HMA_KV_BF16) {
        const uint4 p = pack_row(x);
        r.w[0] = p.x; r.w[1] = p.y; r.w[2] = p.z; r.w[3] = p.w;
    } else {
        uint32_t e[8], E = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = (__float_as_uint(x[i]) >> 23) & 0xFFu;
            if (e[i] == 0xFFu) { bad = true; e[i] = 0; }           // NaN and Inf encode as zero
            E = max(E, e[i]);
        }
        E = max(E, __shfl_xor_sync(0xFFFFFFFFu, E, 1));
        r.E = E;
        // |x| * 2^(top - E) in two exact steps, of which neither leaves the range of fp32
        const int up = (kFmt == HMA_KV_BFP8 ? 133 : 129) - (int)E, one = min(up, 100);
        const float s1 = __uint_as_float((uint32_t)(127 + one) << 23), s2 = __uint_as_float((uint32_t)(127 + up - one) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = e[i] ? min(__float2int_rn(fabsf(x[i]) * s1 * s2), kFmt == HMA_KV_BFP8 ? 127 : 7) : 0;
            const bool neg = __float_as_uint(x[i]) >> 31;
            const int code = kFmt == HMA_KV_BFP8 ? m | (neg ? 0x80 : 0) : neg ? 8 - m : 8 + m;
            r.w[i >> 2] |= (uint32_t)code << (8 * (i & 3));
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
// Thread `i` of kRowThreads writes 16-byte words of the part; rows[t] holds token t's codes (or BF16 values), exps[t] its exponents.
template <int kFmt, bool kV>
__device__ __forceinline__ void store_page(uint8_t *part, const uint8_t (*rows)[kStageStride], const uint8_t (*exps)[8])
{
    constexpr int kHead = kFmt == HMA_KV_BF16 ? 0 : 128;
    constexpr int kWords = (kFmt == HMA_KV_BFP8 ? 2048 : kFmt == HMA_KV_BF16 ? 4096 : 1024) / 16;
    if (kHead && threadIdx.x < 32) {             // exponent bytes, one word a thread
        const int w = threadIdx.x;
        uint32_t v = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int at = 4 * w + b;
            const int tok = kV ? 2 * (at >> 5) + (b & 1) + 8 * (b >> 1) : (at >> 4) + 8 * ((at >> 3) & 1);
            v |= (uint32_t)exps[tok][kV ? (at >> 2) & 7 : at & 7] << (8 * b);
        }
        reinterpret_cast<uint32_t *>(part)[w] = v;
    }
#pragma unroll
    for (int i = threadIdx.x; i < kWords; i += kRowThreads) {
        const int c = i >> 5, g = (i >> 2) & 7, t = i & 3;       // 512-byte piece, lane = 4 * g + t
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (kFmt == HMA_KV_BFP8) {
                if (!kV) w[k] = *reinterpret_cast<const uint32_t *>(&rows[g + 8 * (c & 1)][16 * (4 * (c >> 1) + k) + 4 * t]);
                else {
                    const int ch = 16 * (2 * c + (k >> 1)) + 8 * (k & 1) + g;
                    w[k] = rows[2 * t][ch] | (rows[2 * t + 1][ch] << 8) | (rows[2 * t + 8][ch] << 16) | ((uint32_t)rows[2 * t + 9][ch] << 24);
                }
            } else if constexpr (kFmt == HMA_KV_BF16) {
                if (!kV) w[k] = *reinterpret_cast<const uint32_t *>(&rows[g + 8 * (c & 1)][2 * (16 * (2 * (c >> 1) + (k >> 1)) + 4 * t + 2 * (k & 1))]);
                else {
                    const int ch = 16 * c + 8 * (k & 1) + g, tok = 2 * t + 8 * (k >> 1);
                    w[k] = *reinterpret_cast<const uint16_t *>(&rows[tok][2 * ch]) | ((uint32_t)*reinterpret_cast<const uint16_t *>(&rows[tok + 1][2 * ch]) << 16);
                }
            } else {
                const int j = 4 * c + k;
                if (!kV) {
                    const uint32_t a = *reinterpret_cast<const uint32_t *>(&rows[g][16 * j + 4 * t]), b = *reinterpret_cast<const uint32_t *>(&rows[g + 8][16 * j + 4 * t]);
                    const uint32_t pa = a | (a >> 12), pb = b | (b >> 12);                  // bytes 0 and 1: codes (0, 2) and (1, 3)
                    w[k] = (pa & 0xFFu) | ((pb & 0xFFu) << 8) | ((pa & 0xFF00u) << 8) | ((pb & 0xFF00u) << 16);
                } else {
                    w[k] = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const uint8_t *r = &rows[2 * t + (b >> 1) + 8 * (b & 1)][16 * j + g];
                        w[k] |= (uint32_t)(r[0] | (r[8] << 4)) << (8 * b);
                    }
                }
            }
        }
        *reinterpret_cast<uint4 *>(part + kHead + 16 * i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ---------------------------------------------------------------- the kernel
// kNorm: hma_qk_norm_rope (else hma_kv_append: no row CTAs).  kFmt: format of the cache, kFmtNone without one.
template <bool kF32, int kFmt, bool kNorm, int kRows>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const RowArgs a)
{
    constexpr int kElem = kF32 ? 4 : 2;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
    auto position = [&](int64_t tok) -> int64_t {
        const int64_t p = a.positions[tok];
        if (p >= 0 && p < a.rope_rows) return p;
        if (lane16 == 0) atomicOr(a.flags, HMA_FLAG_BAD_POSITION);
        return 0;                                 // the table's first row: in bounds, and flagged
    };
    auto weights = [&](const uint8_t *w, float (&f)[8]) { if (w) load_row<kF32>(w, lane16, f); };

    if (kNorm && (int64_t)blockIdx.x < a.row_ctas) {
        const int per_token = (a.row_heads + kRows - 1) / kRows;
        const int64_t unit = (int64_t)blockIdx.x * kRowGroups + grp;
        const int64_t tok = unit / per_token;
        const int h0 = (int)(unit - tok * per_token) * kRows;
        const bool live = tok < a.n_tokens;       // a half-warp without work stays for its warp's shuffles
        const int64_t t = live ? tok : a.n_tokens - 1;
        float x[kRows][8], w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        Turn turn;
        const bool keys = h0 >= a.hq;             // the weights of the group's first head; a group that mixes both loads them again
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int h = min(h0 + r, a.row_heads - 1);
            load_row<kF32>(h < a.hq ? a.q + (t * a.k_stride + (int64_t)h * kHeadDim) * kElem : a.k + (t * a.k_stride + (int64_t)(h - a.hq) * kHeadDim) * kElem, lane16, x[r]);
        }
        if (a.half) load_turn(a, position(t), lane16, turn);
        weights(keys ? a.k_weight : a.q_weight, w);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int h = h0 + r;
            if (h == a.hq && r > 0) weights(a.k_weight, w);
            // both half-warps of a warp run the same shuffles, whatever their heads are
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[r][i];
            const bool normed = (h < a.hq ? a.q_weight : a.k_weight) != nullptr;
            norm_row(y, w, a.eps);
            if (normed)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[r][i] = y[i];
            if (a.half) rotate_row(a, lane16, turn, x[r]);
            if (live && h < a.row_heads) {
                uint16_t *o = h < a.hq ? a.q_out + (tok * a.hq + h) * kHeadDim : a.k_out + (tok * a.hkv + h - a.hq) * kHeadDim;
                reinterpret_cast<uint4 *>(o)[lane16] = pack_row(x[r]);
            }
        }
        return;
    }
    if constexpr (kFmt != kFmtNone) {
        __shared__ __align__(16) uint8_t rows[kPageTokens][kStageStride];
        __shared__ uint8_t exps[kPageTokens][8];
        __shared__ int64_t slot[46];              // of tokens base - 15 .. base + 30
        __shared__ int found[2];                  // whole pages: the start before the window that reaches into it, the start inside
        const int64_t unit = (int64_t)blockIdx.x - a.row_ctas;
        const int heads2 = 2 * a.hkv;
        const int64_t base = unit / heads2 * kPageTokens;
        const int hw = (int)(unit % heads2), head = hw >> 1, is_v = hw & 1;
        const int64_t n = a.n_tokens;
        if (threadIdx.x < 46) {
            const int64_t i = base - 15 + threadIdx.x;
            slot[threadIdx.x] = i >= 0 && i < n ? a.slots[i] : -1;
        }
        if (threadIdx.x < 2) found[threadIdx.x] = kNoPage;
        __syncthreads();
        if (threadIdx.x < 31) {                   // does a whole page start at token base - 15 + threadIdx.x?
            const int64_t s = slot[threadIdx.x];
            bool whole = s >= 0 && s + kPageTokens <= a.num_slots && s % kPageTokens == 0;
#pragma unroll
            for (int d = 1; d < kPageTokens; ++d) whole &= slot[threadIdx.x + d] == s + d;
            // whole pages do not overlap, so there is at most one of each kind
            if (whole) found[threadIdx.x >= 15] = (int)threadIdx.x - 15;
        }
        __syncthreads();
        const int before_end = found[0] + kPageTokens, page_at = found[1];        // tokens below before_end are another CTA's
        constexpr size_t kHalf = record_bytes(kFmt) / 2;
        auto part_of = [&](int64_t s) { return a.layer + ((s / kPageTokens * a.hkv + head) * 2 + is_v) * (int64_t)kHalf; };
        float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (kNorm && !is_v) weights(a.k_weight, w);
        bool bad = false;
        // the window's 16 tokens, then those of a page that starts here and ends in the next window
        const int last = page_at == kNoPage ? kPageTokens : page_at + kPageTokens;
        for (int i0 = 0; i0 < last; i0 += kRowGroups) {
            const int i = i0 + grp;
            const int64_t tok = base + i;
            const bool in_page = page_at != kNoPage && i >= page_at && i < page_at + kPageTokens;
            const bool mine = i < kPageTokens && tok < n;
            const int64_t s = mine ? slot[15 + i] : -1;
            const bool single = mine && !in_page && i >= before_end && s != -1;
            const bool place = single && s >= 0 && s < a.num_slots;
            if (single && !place && lane16 == 0) atomicOr(a.flags, HMA_FLAG_BAD_PAGE_INGEST);
            const bool key_row = kNorm && !is_v && a.k_out != nullptr && mine;    // the window's own keys, cached or not
            if (!__any_sync(0xFFFFFFFFu, in_page || place || key_row)) continue;
            const int64_t t = in_page || place || key_row ? tok : base;           // a half-warp without work goes along
            float x[8];
            load_row<kF32>(is_v ? a.v + (t * a.v_stride + (int64_t)head * kHeadDim) * kElem : a.k + (t * a.k_stride + (int64_t)head * kHeadDim) * kElem, lane16, x);
            if (kNorm && !is_v) {
                if (a.k_weight) norm_row(x, w, a.eps);
                if (a.half) {
                    Turn turn;
                    load_turn(a, position(t), lane16, turn);
                    rotate_row(a, lane16, turn, x);
                }
                // the key is what k_out says: rounded to BF16 once, and that value is cached
                const uint4 p = pack_row(x);
                const uint32_t b[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(b[k] << 16); x[2 * k + 1] = __uint_as_float(b[k] & 0xFFFF0000u); }
                if (key_row) reinterpret_cast<uint4 *>(a.k_out + (tok * a.hkv + head) * kHeadDim)[lane16] = p;
            }
            if (!is_v && a.key_layout == HMA_KEYS_INTERLEAVED) interleave_row(lane16, x);
            bool odd = false;
            const Coded r = encode_row<kFmt>(x, odd);
            bad |= odd && (in_page || place);
            const uint32_t other = kFmt == HMA_KV_BFP4 ? __shfl_xor_sync(0xFFFFFFFFu, (lane16 & 1) ? r.w[0] : r.w[1], 1) : 0u;
            if (in_page) {
                uint8_t *d = rows[i - page_at];
                if (kFmt == HMA_KV_BF16) reinterpret_cast<uint4 *>(d)[lane16] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
                else reinterpret_cast<uint2 *>(d)[lane16] = make_uint2(r.w[0], r.w[1]);
                if (kFmt != HMA_KV_BF16 && !(lane16 & 1)) exps[i - page_at][lane16 >> 1] = (uint8_t)r.E;
            } else if (place) {
                if (is_v) store_token<kFmt, true>(part_of(s), (int)(s % kPageTokens), lane16, r, other);
                else store_token<kFmt, false>(part_of(s), (int)(s % kPageTokens), lane16, r, other);
            }
        }
        if (bad) atomicOr(a.flags, HMA_FLAG_BAD_VALUE_ENCODE);
        if (page_at == kNoPage) return;           // the same in every thread
        __syncthreads();
        if (is_v) store_page<kFmt, true>(part_of(slot[15 + page_at]), rows, exps);
        else store_page<kFmt, false>(part_of(slot[15 + page_at]), rows, exps);
    }
}

template <bool kF32, int kFmt, bool kNorm>
static cudaError_t launch_rows(RowArgs &a, cudaStream_t s)
{
    const int64_t cache_ctas = kFmt == kFmtNone ? 0 : (a.n_tokens + kPageTokens - 1) / kPageTokens * 2 * a.hkv;
    if constexpr (kNorm) {
        const bool few = a.n_tokens * a.row_heads <= kFewRows;
        const int64_t per_token = few ? a.row_heads : (a.row_heads + kManyRows - 1) / kManyRows;
        a.row_ctas = (a.n_tokens * per_token + kRowGroups - 1) / kRowGroups;
        const dim3 grid((unsigned)(a.row_ctas + cache_ctas));
        return few ? launch_after(rows_kernel<kF32, kFmt, true, 1>, grid, kRowThreads, 0, s, 1u, a)
                   : launch_after(rows_kernel<kF32, kFmt, true, kManyRows>, grid, kRowThreads, 0, s, 1u, a);
    } else {
        a.row_ctas = 0;
        return launch_after(rows_kernel<kF32, kFmt, false, 1>, dim3((unsigned)cache_ctas), kRowThreads, 0, s, 1u, a);
    }
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
    if (n_tokens > 1 && (k_token_stride < row || v_token_stride < row)) return HMA_ERR_INVALID_ARG;
    if (n_tokens > hma::kMaxRowTokens || k_token_stride > (1 << 30) || v_token_stride > (1 << 30)) return HMA_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens == 0) return HMA_OK;
    if (!k || !v || !slots) return HMA_ERR_INVALID_ARG;
    const int64_t elem = in_dtype == HMA_OUT_F32 ? 4 : 2;
    if (((uintptr_t)k & 15u) || ((uintptr_t)v & 15u) || (n_tokens > 1 && ((k_token_stride * elem & 15) || (v_token_stride * elem & 15)))) return HMA_ERR_ALIGNMENT;
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
    if (n_tokens > 1 && token_stride < row) return HMA_ERR_INVALID_ARG;
    if (n_tokens > hma::kMaxRowTokens || token_stride > (1 << 30)) return HMA_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens == 0) return HMA_OK;
    if (!qkv || !q_out || (!slots && !k_out) || (rotary_dim && (!rope_table || !positions || rope_rows < 1))) return HMA_ERR_INVALID_ARG;
    const int64_t elem = in_dtype == HMA_OUT_F32 ? 4 : 2;
    if (((uintptr_t)qkv & 15u) || (n_tokens > 1 && (token_stride * elem & 15)) || ((uintptr_t)q_weight & 15u) || ((uintptr_t)k_weight & 15u) ||
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
