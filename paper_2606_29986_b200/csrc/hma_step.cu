// What a decode step works out from its request lengths before any layer runs: pages for the new tokens (taken from a
// free list), the block table, the context lengths, and the position and cache slot of every new token.
//
//   sequence b has P = past_lens[b] tokens and gets n = new_lens[b] more; it holds ceil(P / 16) pages and needs
//   ceil((P + n) / 16); the new pages of all sequences, in sequence order, are the free list's entries from its end.
//   token i of the step belongs to the sequence whose [row_starts[b], row_starts[b + 1]) holds i; its position is
//   P + i - row_starts[b], its slot 16 * page + position % 16.
//
// Bound by latency (a few hundred bytes to a few hundred KB).  The lengths of at most 1024 sequences are scanned by every
// CTA for itself, one sequence per thread, so that no CTA waits for another one's scan; the tokens are dealt to the CTAs.
// One launch, except when many tokens (hence many CTAs) meet outputs that share memory with inputs (context lengths over
// past lengths, the free count in place): those are then written by a second, one-CTA launch of the same kernel.
#include "hma_common.cuh"

namespace hma {

constexpr int kStepThreads = 1024;              // one sequence per thread in the scans
constexpr int kStepMaxBatch = 1024;
constexpr int64_t kStepOneCta = 2048;           // two tokens a thread: one CTA
constexpr int64_t kStepCtas = 148;
constexpr int kStepTokens = 1, kStepLengths = 2;
constexpr int kRopeMaxHalf = kHeadDim / 2;

struct StepArgs {
    const int32_t *past, *fresh;
    int batch;
    int32_t *table;
    int max_pages;
    const int32_t *free_pages, *free_count;
    int64_t num_pages;
    int32_t *context, *starts, *positions;
    int64_t *slots;
    int64_t max_tokens;
    int32_t *left;
    uint32_t *flags;
    int parts;                                   // kStepTokens: table entries, positions and slots; kStepLengths: the rest, by CTA 0
};

// Exclusive prefix over the CTA's threads of two counts, and both totals.
__device__ __forceinline__ void scan2(int64_t a, int64_t b, int64_t *scratch, int64_t &ea, int64_t &eb, int64_t &ta, int64_t &tb)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t ia = a, ib = b;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t va = __shfl_up_sync(0xFFFFFFFFu, ia, d), vb = __shfl_up_sync(0xFFFFFFFFu, ib, d);
        if (lane >= d) { ia += va; ib += vb; }
    }
    if (lane == 31) { scratch[warp] = ia; scratch[32 + warp] = ib; }
    __syncthreads();
    if (warp == 0) {
        int64_t wa = scratch[lane], wb = scratch[32 + lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t va = __shfl_up_sync(0xFFFFFFFFu, wa, d), vb = __shfl_up_sync(0xFFFFFFFFu, wb, d);
            if (lane >= d) { wa += va; wb += vb; }
        }
        scratch[lane] = wa; scratch[32 + lane] = wb;
    }
    __syncthreads();
    ea = ia - a + (warp ? scratch[warp - 1] : 0);
    eb = ib - b + (warp ? scratch[32 + warp - 1] : 0);
    ta = scratch[31]; tb = scratch[63];
}

__global__ void __launch_bounds__(kStepThreads) step_tables_kernel(const StepArgs a)
{
    __shared__ int64_t scratch[64];
    __shared__ int start[kStepMaxBatch + 1], before[kStepMaxBatch + 1], past[kStepMaxBatch], held[kStepMaxBatch];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int b = threadIdx.x, B = a.batch;
    const int64_t P = b < B ? a.past[b] : 0, n = b < B ? a.fresh[b] : 0;
    const int64_t count = *a.free_count;
    const bool bad = P < 0 || n < 0 || P + n > (int64_t)a.max_pages * kPageTokens;
    const int64_t h = bad ? 0 : (P + kPageTokens - 1) / kPageTokens, grow = bad ? 0 : (P + n + kPageTokens - 1) / kPageTokens - h;
    int64_t e_tok, e_page, tokens, pages;
    scan2(bad ? 0 : n, grow, scratch, e_tok, e_page, tokens, pages);
    const bool bad_lengths = __syncthreads_or(bad) || tokens > a.max_tokens;
    const bool no_pages = !bad_lengths && (count < 0 || count > a.num_pages || pages > count);
    const bool refused = bad_lengths || no_pages;
    if (!refused) {                              // every number fits an int here: at most max_tokens tokens, num_pages pages
        if (b < B) { start[b] = (int)e_tok; before[b] = (int)e_page; past[b] = (int)P; held[b] = (int)h; }
        if (b == B - 1) { start[B] = (int)tokens; before[B] = (int)pages; }
    }
    __syncthreads();
    // the sequence that holds entry x of an exclusive prefix (the last one that starts at or before it)
    auto owner = [&](const int *prefix, int x) {
        int lo = 0, hi = B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (prefix[mid] <= x) lo = mid; else hi = mid - 1;
        }
        return lo;
    };
    const int64_t first = (int64_t)blockIdx.x * kStepThreads + threadIdx.x, step = (int64_t)gridDim.x * kStepThreads;
    if (!refused && (a.parts & kStepTokens))
        for (int64_t k = first; k < pages; k += step) {
            const int s = owner(before, (int)k);
            a.table[(int64_t)s * a.max_pages + held[s] + ((int)k - before[s])] = a.free_pages[count - 1 - k];
        }
    for (int64_t i = first; i < ((a.parts & kStepTokens) ? a.max_tokens : 0); i += step) {
        int pos = 0;
        int64_t slot = -1;                        // behind the last sequence: no token
        if (!refused && i < tokens) {
            const int s = owner(start, (int)i);
            pos = past[s] + ((int)i - start[s]);
            const int p = pos / kPageTokens;
            // a page that the sequence held before is in the table; a new one comes from the free list, so that nobody
            // waits for the entry to be written
            const int64_t page = p < held[s] ? a.table[(int64_t)s * a.max_pages + p] : a.free_pages[count - 1 - (before[s] + p - held[s])];
            slot = page < 0 ? -2 : page * kPageTokens + pos % kPageTokens;      // a table entry that names no page: not a place either
        }
        a.positions[i] = pos;
        a.slots[i] = slot;
    }
    // (only CTA 0 has read what these may replace, or nothing is replaced)
    if ((a.parts & kStepLengths) && blockIdx.x == 0) {
        if (b < B) {
            a.context[b] = (int32_t)(refused ? P : P + n);
            a.starts[b] = refused ? 0 : (int32_t)e_tok;
        }
        if (b == 0) {
            a.starts[B] = refused ? 0 : (int32_t)tokens;
            *a.left = (int32_t)(refused ? count : count - pages);
            if (refused) atomicOr(a.flags, bad_lengths ? HMA_FLAG_BAD_LENGTHS : HMA_FLAG_NO_PAGES);
        }
    }
}

// Pages of finished sequences back onto the free list, in sequence order, each sequence's first page first; table entries that
// name no page (given up behind a window, say) are passed over.  One CTA: a batch loses a few sequences per step.
__global__ void __launch_bounds__(kStepThreads) release_pages_kernel(const int32_t *finished, int32_t *context, int batch, int32_t *table,
                                                                     int max_pages, int32_t *free_pages, int32_t *free_count,
                                                                     int64_t num_pages, uint32_t *flags)
{
    __shared__ int64_t scratch[64];
    __shared__ int before[kStepMaxBatch + 1];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int b = threadIdx.x;
    const int64_t T = b < batch ? context[b] : 0, count = *free_count;
    const bool bad = T < 0 || T > (int64_t)max_pages * kPageTokens, gone = b < batch && finished[b] != 0;
    const int64_t held = bad || !gone ? 0 : (T + kPageTokens - 1) / kPageTokens;
    int64_t e, unused, pages, none;
    scan2(held, 0, scratch, e, unused, pages, none);
    const bool bad_lengths = __syncthreads_or(bad && gone);
    if (!bad_lengths) {                          // (the same in every thread)
        if (b < batch) before[b] = (int)e;
        if (b == 0) before[batch] = (int)pages;
    }
    __syncthreads();
    auto entry = [&](int64_t k) {                // of the k-th page of the finished sequences
        int lo = 0, hi = batch - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (before[mid] <= k) lo = mid; else hi = mid - 1;
        }
        return table + (int64_t)lo * max_pages + (k - before[lo]);
    };
    auto page_at = [&](int64_t k) {              // -1: none (behind the last one, or given up earlier)
        const int32_t page = k < pages ? *entry(k) : -1;
        return page >= 0 && page < num_pages ? page : -1;
    };
    bool refused = bad_lengths || count < 0 || pages > INT32_MAX;
    if (!refused && count + pages > num_pages) { // entries that name no page may make the difference: count the ones that do
        int64_t named = 0;
        for (int64_t c = 0; c < pages; c += kStepThreads) named += __syncthreads_count(page_at(c + threadIdx.x) >= 0);
        refused = count + named > num_pages;
    }
    if (refused) {                               // the same in every thread
        if (b == 0) atomicOr(flags, bad_lengths ? HMA_FLAG_BAD_LENGTHS : HMA_FLAG_NO_PAGES);
        return;
    }
    int64_t end = count;
    for (int64_t c = 0; c < pages; c += kStepThreads) {
        const int64_t k = c + threadIdx.x;
        const int32_t page = page_at(k);
        int64_t place = threadIdx.x, unused2, named = __syncthreads_count(page >= 0);
        if (named < min((int64_t)kStepThreads, pages - c)) {
            scan2(page >= 0, 0, scratch, place, unused2, named, none);
            __syncthreads();                     // before the next round's scan writes its scratch array
        }
        if (page >= 0) free_pages[end + place] = page;
        if (k < pages) *entry(k) = -1;
        end += named;
    }
    __syncthreads();
    if (gone) context[b] = 0;
    if (b == 0) *free_count = (int32_t)end;
}

// cos and sin of position * inv_freq[i], formed in 64 bits: a 32-bit product is off by up to position * 2^-25 radians
// (4e-3 at position 131072), which the rotation would carry into every key.
struct RopeFreqs { double f[kRopeMaxHalf]; };
__global__ void __launch_bounds__(256) rope_table_kernel(const RopeFreqs fr, int half, int64_t first_pos, int64_t n_pos, double scale, float *table)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_pos * half; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t p = i / half;
        const int k = (int)(i - p * half);
        double s, c;
        sincos((double)(first_pos + p) * fr.f[k], &s, &c);
        table[p * 2 * half + k] = (float)(c * scale);
        table[p * 2 * half + half + k] = (float)(s * scale);
    }
}

}  // namespace hma

extern "C" hma_status_t hma_step_tables(const hma_cache_t *cache, const int32_t *past_lens, const int32_t *new_lens, int32_t batch,
                                        int32_t *block_table, int32_t max_pages_per_seq, const int32_t *free_pages,
                                        const int32_t *free_count, int32_t *context_lens, int32_t *row_starts, int32_t *positions,
                                        int64_t *slots, int64_t max_tokens, int32_t *free_count_out, void *stream)
{
    if (!cache || batch < 0 || max_pages_per_seq < 0 || max_tokens < 0) return HMA_ERR_INVALID_ARG;
    if (!hma::on_cache_device(cache)) return HMA_ERR_INVALID_ARG;
    if (batch > hma::kStepMaxBatch || max_pages_per_seq > (1 << 26) || max_tokens > (1 << 30) || cache->desc.num_pages > INT32_MAX)
        return HMA_ERR_UNSUPPORTED_SHAPE;
    if (!row_starts || !free_count || !free_count_out || (max_tokens && (!positions || !slots))) return HMA_ERR_INVALID_ARG;
    if (batch && (!past_lens || !new_lens || !context_lens || !block_table || !free_pages)) return HMA_ERR_INVALID_ARG;
    hma::StepArgs a{past_lens, new_lens, batch, block_table, max_pages_per_seq, free_pages, free_count, cache->desc.num_pages,
                    context_lens, row_starts, positions, slots, max_tokens, free_count_out, cache->flags, hma::kStepTokens | hma::kStepLengths};
    if (max_tokens > hma::kStepOneCta) {
        const int64_t ctas = (max_tokens + hma::kStepThreads - 1) / hma::kStepThreads;
        const bool in_place = context_lens == past_lens || free_count_out == free_count;
        if (in_place) a.parts = hma::kStepTokens;
        HMA_CUDA_OK(hma::launch_after(hma::step_tables_kernel, dim3((unsigned)(ctas < hma::kStepCtas ? ctas : hma::kStepCtas)), hma::kStepThreads, 0, (cudaStream_t)stream, a));
        hma::count_launch();
        if (!in_place) return HMA_OK;
        a.parts = hma::kStepLengths;
    }
    HMA_CUDA_OK(hma::launch_after(hma::step_tables_kernel, dim3(1), hma::kStepThreads, 0, (cudaStream_t)stream, a));
    hma::count_launch();
    return HMA_OK;
}

extern "C" hma_status_t hma_release_pages(const hma_cache_t *cache, const int32_t *finished, int32_t *context_lens, int32_t batch,
                                          int32_t *block_table, int32_t max_pages_per_seq, int32_t *free_pages, int32_t *free_count,
                                          void *stream)
{
    if (!cache || batch < 0 || max_pages_per_seq < 0) return HMA_ERR_INVALID_ARG;
    if (!hma::on_cache_device(cache)) return HMA_ERR_INVALID_ARG;
    if (batch > hma::kStepMaxBatch || max_pages_per_seq > (1 << 26) || cache->desc.num_pages > INT32_MAX) return HMA_ERR_UNSUPPORTED_SHAPE;
    if (batch == 0) return HMA_OK;
    if (!finished || !context_lens || !block_table || !free_pages || !free_count) return HMA_ERR_INVALID_ARG;
    HMA_CUDA_OK(hma::launch_after(hma::release_pages_kernel, dim3(1), hma::kStepThreads, 0, (cudaStream_t)stream, finished, context_lens,
                                  (int)batch, block_table, (int)max_pages_per_seq, free_pages, free_count, cache->desc.num_pages, cache->flags));
    hma::count_launch();
    return HMA_OK;
}

extern "C" hma_status_t hma_rope_table(const double *inv_freq, int32_t rotary_dim, int64_t first_pos, int64_t n_pos, double scale,
                                       float *table, void *stream)
{
    if (!inv_freq || first_pos < 0 || n_pos < 0) return HMA_ERR_INVALID_ARG;
    if (rotary_dim < 16 || rotary_dim > hma::kHeadDim || rotary_dim % 16 || first_pos > INT32_MAX || n_pos > (int64_t)INT32_MAX + 1 - first_pos)
        return HMA_ERR_UNSUPPORTED_SHAPE;
    if (n_pos == 0) return HMA_OK;
    if (!table) return HMA_ERR_INVALID_ARG;
    if ((uintptr_t)table & 15u) return HMA_ERR_ALIGNMENT;
    hma::RopeFreqs fr = {};
    for (int i = 0; i < rotary_dim / 2; ++i) fr.f[i] = inv_freq[i];
    int64_t blocks = (n_pos * (rotary_dim / 2) + 255) / 256;
    if (blocks > 148 * 8) blocks = 148 * 8;
    HMA_CUDA_OK(hma::launch_after(hma::rope_table_kernel, dim3((unsigned)blocks), 256, 0, (cudaStream_t)stream, fr, (int)(rotary_dim / 2),
                                  first_pos, n_pos, scale, table));
    hma::count_launch();
    return HMA_OK;
}
