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

// Exclusive prefix sum over the block; *total: the sum.  Both barriers inside.
__device__ __forceinline__ int block_scan(int x, int* warp_sums, int* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int in = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, in, o);
        if (lane >= o) in += y;
    }
    if (lane == 31) warp_sums[warp] = in;
    __syncthreads();
    int s = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    *total = __shfl_sync(0xffffffffu, s, 31);
    const int before = __shfl_sync(0xffffffffu, s, warp) - warp_sums[warp];
    __syncthreads();
    return before + in - x;
}

// One CTA per sequence.  The weight of the last page that stays is found digit by digit (8 bits at a time, from the top): a
// histogram of the digit among the pages that share the digits found so far.  Then one pass in page order moves what stays
// forward; a chunk is read before anything of it is written and nothing is written ahead of the reading, so the outputs may
// be the inputs.
__global__ void __launch_bounds__(EVICT_THREADS)
cache_evict_kernel(const CacheView c, const float* weight, int keep, int first, int last, int* table_out, int* lens_out,
                   float* weight_out, int* __restrict__ freed, int* __restrict__ n_freed)
{
    __shared__ int hist[256], sums[32], digit, rest;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x, tid = threadIdx.x;
    const long long row = (long long)b * c.max_pages;
    const int raw_len = c.lens[b];
    const bool bad = raw_len < 0 || raw_len > (long long)c.max_pages * 64;
    const int np = bad ? 0 : (raw_len + 63) >> 6;
    const int lo = first, hi = np - last;                            // pages [lo, hi) may go
    const bool evict = np > keep;
    uint32_t bar = 0;                                                // order of the last page that stays
    int ties = 0;                                                    // pages of that order that stay
    if (evict) {
        ties = keep - first - last;
        uint32_t mask = 0;
        for (int sh = 24; sh >= 0 && ties > 0; sh -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int i = lo + tid; i < hi; i += EVICT_THREADS) {
                const uint32_t o = order_of(weight[row + i]);
                if ((o & mask) == bar) atomicAdd(&hist[o >> sh & 255], 1);
            }
            __syncthreads();
            int total;
            const int mine = tid < 256 ? hist[255 - tid] : 0;        // largest digit first
            const int before = block_scan(mine, sums, &total);
            if (tid < 256 && before < ties && before + mine >= ties) {
                digit = 255 - tid;
                rest = ties - before;
            }
            __syncthreads();
            bar |= (uint32_t)digit << sh;
            mask |= 255u << sh;
            ties = rest;
            __syncthreads();
        }
        if (keep == first + last) { bar = 0xFFFFFFFFu; ties = 0; }
    }
    int kept = 0, gone = 0, equal = 0;                               // so far
    const int n = bad ? c.max_pages : np;
    for (int i0 = 0; i0 < n; i0 += EVICT_THREADS) {
        const int i = i0 + tid;
        const bool in = i < n;
        const int page = in ? c.table[row + i] : 0;
        const float w = in ? weight[row + i] : 0.f;
        const bool middle = evict && i >= lo && i < hi;
        const uint32_t o = order_of(w);
        int total;
        const bool tie = in && middle && o == bar;
        const int nth = equal + block_scan(tie, sums, &total);
        equal += total;
        const bool stays = in && (!middle || o > bar || (tie && nth < ties));
        const int at = kept + block_scan(stays, sums, &total);
        const int chunk = min(EVICT_THREADS, n - i0);
        if (stays) {
            table_out[row + at] = page;
            weight_out[row + at] = w;
        } else if (in) {
            freed[row + gone + (tid - (at - kept))] = page;
        }
        kept += total;
        gone += chunk - total;
    }
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
