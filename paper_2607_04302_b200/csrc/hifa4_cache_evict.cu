// Eviction of whole pages from block tables by accumulated attention weight.
#include "hifa4_cache.cuh"

namespace hifa4 {

constexpr int EVICT_THREADS = 1024;

// Weights as integers of the same order: -0 equals +0, a NaN lies below everything.
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0;
    const uint32_t b = __float_as_uint(w + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive prefix sum over the block of two 16-bit counts in a word; *total: the sums.  `sums`: 32 words that the call before the last
// one used (one barrier per call).
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* sums, uint32_t* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t in = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, in, o);
        if (lane >= o) in += y;
    }
    if (lane == 31) sums[warp] = in;
    __syncthreads();
    const uint32_t mine = sums[lane];
    uint32_t s = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    *total = __shfl_sync(0xffffffffu, s, 31);
    return __shfl_sync(0xffffffffu, s - mine, warp) + in - x;
}

// One CTA per sequence.  The weight of the last page that stays is found digit by digit (8 bits at a time, from the top): a
// histogram of the digit among the pages that share the digits found so far, searched by one warp (two bits at a time by counting
// against thresholds takes more barriers: 18.4 against 8.1 us for 256 sequences of 2048 pages), until all pages that share them
// stay (without that end 8.7; 4 sequences of 70 pages 5.4 instead of 4.0).  Then one pass in page order moves what stays forward; a
// chunk is read before anything of it is written and nothing is written ahead of the reading, so the outputs may be the inputs.
constexpr int EVICT_HELD = 4;                                        // orders that a thread holds; longer tables are read again
__global__ void __launch_bounds__(EVICT_THREADS)
cache_evict_kernel(const CacheView c, const float* weight, int keep, int first, int last, int* table_out, int* lens_out,
                   float* weight_out, int* __restrict__ freed, int* __restrict__ n_freed)
{
    __shared__ uint32_t scan_sums[2][32];
    __shared__ int hist[4][256], found[3];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long row = (long long)b * c.max_pages;
    const int raw_len = c.lens[b];
    const bool bad = raw_len < 0 || raw_len > (long long)c.max_pages * 64;
    const int np = bad ? 0 : (raw_len + 63) >> 6;
    const int lo = first, hi = np - last;                            // pages [lo, hi) may go
    const bool evict = np > keep;
    uint32_t bar = 0;                                                // order of the last page that stays
    int ties = 0;                                                    // pages of that order that stay
    if (evict) {
        const int stay = keep - first - last;
        uint32_t held[EVICT_HELD];
#pragma unroll
        for (int i = 0; i < EVICT_HELD; ++i) {
            const int at = lo + tid + i * EVICT_THREADS;
            held[i] = at < hi ? order_of(weight[row + at]) : 0;
        }
        ties = stay;
        hist[tid >> 8][tid & 255] = 0;
        if (stay == 0) bar = 0xFFFFFFFFu;                            // above the order of any number
        for (int sh = 24; sh >= 0 && stay > 0; sh -= 8) {
            int* const h = hist[sh >> 3];
            const uint32_t mask = sh == 24 ? 0u : 0xFFFFFFFFu << (sh + 8);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EVICT_HELD; ++i)
                if (lo + tid + i * EVICT_THREADS < hi && (held[i] & mask) == bar) atomicAdd(&h[held[i] >> sh & 255], 1);
            for (int at = lo + tid + EVICT_HELD * EVICT_THREADS; at < hi; at += EVICT_THREADS) {
                const uint32_t o = order_of(weight[row + at]);
                if ((o & mask) == bar) atomicAdd(&h[o >> sh & 255], 1);
            }
            __syncthreads();
            if (warp == 0) {                                         // lane: eight digits, the largest ones in lane 0
                int n[8], sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += n[i] = h[255 - 8 * lane - i];
                int in = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, in, o);
                    if (lane >= o) in += y;
                }
                int before = in - sum;
                if (before < ties && in >= ties) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (before < ties && before + n[i] >= ties) {
                            found[0] = 255 - 8 * lane - i;
                            found[1] = ties - before;
                            found[2] = n[i];
                        }
                        before += n[i];
                    }
                }
            }
            __syncthreads();
            bar |= (uint32_t)found[0] << sh;
            ties = found[1];
            if (found[2] == ties && bar) {                           // all pages that share these digits stay: no need for the others
                --bar;
                ties = 0;
                break;
            }
        }
    }
    int strict = 0, equal = 0;                                       // pages before the chunk that stay for sure; of the order `bar`
    const int n = bad ? c.max_pages : np;
    for (int i0 = 0, turn = 0; i0 < n; i0 += EVICT_THREADS, turn ^= 1) {
        const int i = i0 + tid;
        const bool in = i < n;
        const int page = in ? c.table[row + i] : 0;
        const float w = in ? weight[row + i] : 0.f;
        const bool middle = evict && i >= lo && i < hi;
        const uint32_t o = order_of(w);
        const bool sure = in && (!middle || o > bar), tie = in && middle && o == bar;
        uint32_t total;
        const uint32_t before = block_scan((uint32_t)sure << 16 | (uint32_t)tie, scan_sums[turn], &total);
        const int tied = equal + (int)(before & 0xFFFF);
        const int at = strict + (int)(before >> 16) + min(tied, ties);       // pages before this one that stay
        if (sure || (tie && tied < ties)) {
            table_out[row + at] = page;
            weight_out[row + at] = w;
        } else if (in) {
            freed[row + i - at] = page;
        }
        strict += (int)(total >> 16);
        equal += (int)(total & 0xFFFF);
    }
    const int kept = strict + min(equal, ties), gone = n - kept;
    __syncthreads();
    for (int i = kept + tid; i < c.max_pages; i += EVICT_THREADS) {
        table_out[row + i] = -1;
        weight_out[row + i] = 0.f;
    }
    for (int i = gone + tid; i < c.max_pages; i += EVICT_THREADS) freed[row + i] = -1;
    if (tid == 0) {
        lens_out[b] = raw_len - 64 * gone;
        n_freed[b] = gone;
        if (bad) c.invalid();
    }
}

cudaError_t launch_cache_evict(const CacheView& c, const float* weight, int keep, int first, int last, int* table_out,
                               int* lens_out, float* weight_out, int* freed, int* n_freed, cudaStream_t st)
{
    return launch_dependent(cache_evict_kernel, (unsigned)c.B, EVICT_THREADS, 0, st, c, weight, keep, first, last, table_out, lens_out,
                            weight_out, freed, n_freed);
}

}  // namespace hifa4
