// What the kernels of the paged HIF4 cache share: layout of a page, checks of lengths and page numbers, arguments.
#pragma once
#include "hifa4_internal.h"
#include "hifa4_device.cuh"

namespace hifa4 {

// Byte offsets in a head's part of a page (see include/hifa4.h).
template <int D> struct Page {
    static constexpr int NG = D / 64;                          // groups per token of K
    static constexpr int K_CODES = 0, K_SHIFTS = 32 * D, K_SCALES = 36 * D;
    static constexpr int HALF = 37 * D;                        // V's half repeats the layout of K's
    static constexpr int BYTES = 74 * D;
};

struct CacheView {
    uint8_t* pages;                    // [n_pages][Hkv][74 d]
    uint16_t* v_tail;                  // [n_tails][Hkv][64][d] or null
    int n_pages, n_tails, Hkv;
    int B, max_pages;
    const int *table, *lens, *slots;
    int* d_status;
    // Tokens of sequence b; -1 where the length is out of range.
    __device__ __forceinline__ int len(int b) const
    {
        const int n = __ldg(lens + b);
        return n < 0 || n > (long long)max_pages * 64 ? -1 : n;
    }
    // Pages of sequence b (none where the length is out of range).
    __device__ __forceinline__ int n_pages_of(int b) const { return (max(len(b), 0) + 63) >> 6; }
    // Physical page, -1 where it is out of range.
    __device__ __forceinline__ int page(int b, int p) const
    {
        const int g = __ldg(table + (long long)b * max_pages + p);
        return g < 0 || g >= n_pages ? -1 : g;
    }
    // The status word keeps the first code, but an expired wait outweighs a bad length, page or slot.
    __device__ __forceinline__ void invalid() const
    {
        if (d_status) atomicCAS(d_status, 0, HIFA4_ERR_INVALID_ARG);
    }
    __device__ __forceinline__ void timed_out() const
    {
        if (d_status) atomicMax(d_status, HIFA4_ERR_TIMEOUT);
    }
};

__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t c)
{
    uint32_t r;                        // (from the operators the compiler forms twice as many instructions)
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(mask), "r"(c));
    return r;
}
// The scale S of code c as a BF16 number in both halves.
__device__ __forceinline__ uint32_t scale_pair(uint32_t c) { return ((c << 5) + (79u << 7)) * 0x10001u; }
// A group's shift word, turned so that the shifts of unit u (bits 2 u and 16 + 2 u) come to lie in bits 7-8 and 23-24.
__device__ __forceinline__ uint32_t shifts_of_unit(uint32_t w, int u) { return __funnelshift_l(w, w, 7 - 2 * u); }
// One word of codes -> 8 BF16 values, pairs (nibble i, nibble i + 4).  y: see shifts_of_unit; s2: see scale_pair.
// big = 32 * 2^shift; with a nibble in the mantissa (34 + code / 4) * 2^shift; times S less 34 * 2^shift * S (7 significant bits): exact.
__device__ __forceinline__ void hif4_word_values(uint32_t w, uint32_t y, uint32_t s2, uint32_t (&r)[4])
{
    const uint32_t big = and_or(y, 0x01800180u, 0x42004200u);
    uint32_t sub = and_or(y, 0x01800180u, 0xC208C208u);                     // -34 * 2^shift
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(sub) : "r"(sub), "r"(s2));
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = bf2_fma(and_or(w >> (4 * i), 0x000F000Fu, big), s2, sub);
}

struct Strides { long long b, h, t; };

// Query heads sorted by KV head; unit u = (KV head, rows of a block).  A row is (query head, query token).
struct CacheUnits {
    uint8_t head[HIFA4_MAX_HEADS];     // query heads in the order of their KV heads
    short first[HIFA4_MAX_HEADS + 1];  // first entry of `head` of each KV head
};

struct DecodeArgs {
    CacheView cache;
    CacheUnits units;
    const void* q;
    Strides qs;
    const float* s;                    // [Hkv,d] or null
    int Hq, N, causal, out_dtype;
    int blocks;                        // row blocks per KV head
    uint32_t one;                      // 1, as a value that the compiler does not know
    float scale_log2;                  // softmax scale times log2(e)
    void* out;                         // [B,Hq,N,d]
    float* lse;                        // [B,Hq] or null
    const float* weight;
    float* weight_out;                 // [B][max_pages] or null
    float* first;                      // first pieces of warps that go on to other segments: [DECODE_CTAS * warps][rows (d + 2)]
    float* part_o;                     // partial sums of segments that cross CTAs: [2 * DECODE_CTAS][rows][d]
    float2* part_ml;                   // their references and sums of p: [2 * DECODE_CTAS][rows]
    int4* begun;                       // [DECODE_CTAS]: sequence, unit and last CTA of the segment that goes on behind a CTA, -1: none
    int2* seg_ctas;                    // [B][units]: first and last CTA of each segment (page weights only)
    float2* final_ml;                  // the same of whole rows, [B][Hq] (page weights only)
    float2* page_ml;                   // the same of pages, [B][Hq][max_pages] (page weights only)
};

struct TileArgs {
    CacheView cache;
    CacheUnits units;
    const void* q;
    Strides qs;
    const float* s;
    int Hq, N, causal, out_dtype;
    int items;                         // row blocks per KV head
    int full, splits;                  // blocks [0, full) have a CTA each, the others `splits` CTAs
    float scale_log2;
    void* out;
    float* part_o;                     // [block - full][tile][split][128][d]
    float2* part_ml;
};

cudaError_t launch_cache_append(int dtype, int d, const CacheView& c, int n, const int* n_new, const void* k, Strides ks,
                                const void* v, Strides vs, const float* inv_s, cudaStream_t st);
cudaError_t launch_cache_read(int d, const CacheView& c, int n, const int* start, int out_dtype, void* k, void* v,
                              cudaStream_t st);
cudaError_t launch_cache_evict(const CacheView& c, const float* weight, int keep, int first, int last, int* table_out,
                               int* lens_out, float* weight_out, int* freed, int* n_freed, cudaStream_t st);
constexpr int DECODE_CTAS = 148;       // one per SM; part of the workspace's size
// Whether CTAs c0 to c1 can hold a segment.  What a decode kernel that gave up left unwritten in the workspace is arbitrary.
__host__ __device__ inline bool segment_recorded(int c0, int c1) { return c0 >= 0 && c0 <= c1 && c1 < DECODE_CTAS; }
// Rows per block for a problem with `rows` rows per KV head at most.
int decode_block_rows(int d, int rows);
size_t decode_first_floats(int d, int block_rows);
cudaError_t launch_cache_decode(int dtype, int d, int block_rows, const DecodeArgs& a, cudaStream_t st);
cudaError_t launch_cache_decode_selftest(const DecodeArgs& a, cudaStream_t st);          // BF16, d = 128, 8 rows

// Query rows that a CTA of the tensor-memory kernel takes.
int attention_tile_rows(int dtype, int d);
cudaError_t launch_cache_attention(int dtype, int d, const TileArgs& a, cudaStream_t st);
cudaError_t launch_cache_attention_selftest(const TileArgs& a, cudaStream_t st);         // BF16, d = 128

}  // namespace hifa4
