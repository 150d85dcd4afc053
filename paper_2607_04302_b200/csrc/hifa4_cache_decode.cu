// Attention of a few query rows per KV head over the paged HIF4 cache, split over the caches' lengths and joined.
//
//   S = q~ K^T scale,  m = running max,  p = exp2(S log2e - m + 15),  l = sum p,  O = p V / l
//
// Work: the (sequence, block of query rows of a KV head, page) triples of all sequences, in this order, are dealt out to the
// consumer warps of one CTA per SM in equal contiguous ranges, whatever the sequences' lengths.  A consumer takes whole pages on
// its own: it forms S of the page's 64 tokens, its softmax and O, all in registers, without any exchange between
// warps.  One more warp loads the pages (bulk copies, a lane per consumer).  The pages of one (sequence, block) that a
// range holds are a piece of its segment; pieces that warps of one CTA share are joined in shared memory, those that CTAs share by
// a second, small kernel.
//
// Products run on mma.sync m16n8k16 with the cache as the 16-row operand, tokens (S) or channels (O) its rows, and query rows as the
// 8 columns: an operand of 5 or 6 query rows would leave a 128-row tcgen05 tile nearly empty, and its other operand would have to
// pass through shared memory as 16-bit values, four times the bytes of the codes.  Here codes become FP16 operands in
// registers (code * 2^shift, at most 28 in magnitude, exact); the scale of a group multiplies the FP32 sums of the
// group's products, per token for S, per channel for O.  Any order of the contraction index will do as long as both operands
// agree on it, so each lane takes whole 8-code words.
#include "hifa4_cache.cuh"

namespace hifa4 {

using namespace ptx;

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// a + c in the multiply-add pipe (one: 1, which the compiler must not know): the logic pipe, half as wide, is the busier one.
__device__ __forceinline__ uint32_t add_mad(uint32_t a, uint32_t one, uint32_t c)
{
    uint32_t r;
    asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(one), "r"(c));
    return r;
}
// Eight codes of a word as four packed pairs (nibble i, nibble i + 4) of code * 2^shift / 2 in FP16.  y holds the two shifts in the
// low exponent bits (10-11 and 26-27); its other bits do not matter.  A nibble lands in the mantissa of a power of two whose
// exponent's low two bits are clear, so one logic operation with y forms that number times 2^shift; what the number is too large
// by is subtracted.  All steps are exact.
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t y, uint32_t one, uint32_t (&r)[4])
{
    const uint32_t big = and_or(y, 0x0C000C00u, 0x60006000u);         // 512 * 2^shift; with a nibble: (512 + nibble / 2) * 2^shift
    const uint32_t sub = add_mad(big, one, 0x80088008u);              // -516 * 2^shift
    const uint32_t sub16 = add_mad(big, one, 0x70807080u);            // -36 * 2^shift
    const uint32_t v = w >> 8, sixteenth = 0x2C002C00u;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r[0]) : "r"(and_or(w, 0x000F000Fu, big)), "r"(sub));
    r[1] = h2_fma(and_or(w, 0x00F000F0u, big), sixteenth, sub16);     // (512 + 8 nibble) * 2^shift / 16
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r[2]) : "r"(and_or(v, 0x000F000Fu, big)), "r"(sub));
    r[3] = h2_fma(and_or(v, 0x00F000F0u, big), sixteenth, sub16);
}
// S/4 of scale code c, times the 2 that unpack8 leaves out.
__device__ __forceinline__ float half_scale(uint32_t c) { return __uint_as_float((c << 21) + (78u << 23)); }
// Shift word of a group, turned so that the shifts of unit 2 t come to lie where unpack8 wants them (bits 2 u, 16 + 2 u of the
// word belong to unit u); unit 2 t + 1: two bits further down.
__device__ __forceinline__ uint32_t turn(uint32_t w, int t) { return __funnelshift_l(w, w, 10 - 4 * t); }

__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }

// NT: 8-row column tiles of query rows.  A consumer has room for one page; the K half is loaded again while V is multiplied, and
// the other way round.  The query operands wait in shared memory while V is multiplied.
template <int D, int NT> struct DecodeCfg {
    static constexpr int W = D == 256 ? 7 : NT == 1 ? 15 : D == 128 ? 7 : 11;   // consumers
    static constexpr int THREADS = (W + 1) * 32;
    static constexpr int ROWS = 8 * NT;
    static constexpr int PV_ROW = 36;                                    // words of P per query row: 32 and 4 against bank conflicts
    static constexpr int PIECE = ROWS * (D + 2);                         // floats of a partial result: O [ROWS][D], then (m, l) [ROWS]
    static constexpr int K_OFF = 0, V_OFF = Page<D>::HALF, P_OFF = Page<D>::BYTES, Q_OFF = P_OFF + NT * 8 * PV_ROW * 4;
    static constexpr int PER_WARP = Q_OFF + ROWS * D * 2;
    static constexpr int BAR_OFF = W * PER_WARP;                         // per consumer: K landed, V landed, K read, V read
    static constexpr int SMEM = BAR_OFF + W * 32 + 64;
    static_assert(PER_WARP % 16 == 0 && Page<D>::HALF % 16 == 0 && PIECE * 4 <= PER_WARP && SMEM <= 227 * 1024 - 2048, "shared memory");
};

// A position in the list of work: page `p` of `np` of unit `u` of sequence `b`.
struct Cursor {
    int b, u, p, np;
};

// Pages of sequences [0, upto), times the units per sequence.  Whole block; all threads get the sum.
__device__ __forceinline__ long long pages_before(const CacheView& c, int upto, long long* scratch)
{
    long long s = 0;
    for (int b = threadIdx.x; b < upto; b += blockDim.x) s += c.n_pages_of(b);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    long long t = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) t += scratch[w];
    return t;
}

// Where page `at` of the list of work is (at is less than the list's length).  Whole warp.
__device__ __forceinline__ Cursor locate(const CacheView& c, int U, long long at, int lane)
{
    Cursor cur{0, 0, 0, 1};
    long long before = 0;
    for (int b0 = 0; b0 < c.B; b0 += 32) {
        const int np = b0 + lane < c.B ? c.n_pages_of(b0 + lane) : 0;
        int pre = np;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, pre, o);
            if (lane >= o) pre += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, (before + pre) * U > at);
        if (hit) {
            const int l = __ffs(hit) - 1;
            cur.b = b0 + l;
            cur.np = __shfl_sync(0xffffffffu, np, l);
            before += __shfl_sync(0xffffffffu, pre - np, l);
            break;
        }
        before += __shfl_sync(0xffffffffu, pre, 31);
    }
    const int in = (int)(at - before * U);
    cur.u = in / cur.np;
    cur.p = in % cur.np;
    return cur;
}

__device__ __forceinline__ float warp_max(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// CTAs that take part: every one of them has a page at least.
__device__ __forceinline__ int active_ctas(long long total) { return (int)min((long long)DECODE_CTAS, total); }

__device__ __forceinline__ int units_per_seq(const DecodeArgs& a) { return a.cache.Hkv * a.blocks; }

// Row r of unit u: query head and token; false behind the last row.
template <int ROWS>
__device__ __forceinline__ bool row_of(const DecodeArgs& a, int u, int r, int& head, int& tok)
{
    const int kv = u / a.blocks, i = (u % a.blocks) * ROWS + r;
    const int first = a.units.first[kv], n = (a.units.first[kv + 1] - first) * a.N;
    if (i >= n) return false;
    head = a.units.head[first + i / a.N];
    tok = i % a.N;
    return true;
}

__device__ __forceinline__ void store_out(const DecodeArgs& a, int b, int head, int tok, int D, int ch, float x)
{
    const long long i = (((long long)b * a.Hq + head) * a.N + tok) * D + ch;
    if (a.out_dtype == HIFA4_BF16) ((__nv_bfloat16*)a.out)[i] = __float2bfloat16_rn(x);
    else if (a.out_dtype == HIFA4_F16) ((__half*)a.out)[i] = __float2half_rn(x);
    else ((float*)a.out)[i] = x;
}
__device__ __forceinline__ void store_row_stats(const DecodeArgs& a, int b, int head, int tok, float m, float l)
{
    if (a.lse) a.lse[((long long)b * a.Hq + head) * a.N + tok] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : l == 0.f ? -INFINITY : l;
    if (a.final_ml) a.final_ml[(long long)b * a.Hq + head] = make_float2(m, l);
}

// Factor that takes sums under the reference m to the reference M >= m (both -inf: nothing there).
__device__ __forceinline__ float rebase(float m, float M) { return m == -INFINITY ? 0.f : exp2f(m - M); }

template <typename T, int D, int NT>
__global__ void __launch_bounds__(DecodeCfg<D, NT>::THREADS, 1)
cache_decode_kernel(const __grid_constant__ DecodeArgs a)
{
    using C = DecodeCfg<D, NT>;
    using P = Page<D>;
    constexpr int NG = P::NG, W = C::W, ROWS = C::ROWS;
    constexpr bool BF = sizeof(T) == 2 && !__is_same(T, __half);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long scratch[W + 1];
    __shared__ Cursor begin_of[W];                     // first page of a consumer's range
    __shared__ int pages_of[W];
    __shared__ volatile int page_there[W];             // whether the page in a consumer's buffers exists
    __shared__ volatile int gave_up;
    __shared__ Cursor piece[2 * W];                    // pieces of segments that a consumer shares with others: [2 w] begun before it,
                                                       // [2 w + 1] in it
    __shared__ long long piece_at[2 * W];              // index of the segment's first page in the list of work, -1: no such piece
    __shared__ float* piece_of[2 * W];                 // where it is
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const uint32_t base = smem_u32(smem) + warp * C::PER_WARP;
    const uint32_t kb = base + C::K_OFF, vb = base + C::V_OFF, pbuf = base + C::P_OFF, qbuf = base + C::Q_OFF + 16 * lane;
    const uint32_t bars = smem_u32(smem) + C::BAR_OFF + warp * 32;
    if (tid < 4 * W) mbar_init(smem_u32(smem) + C::BAR_OFF + 8 * tid, 1);
    if (tid < 2 * W) piece_at[tid] = -1;
    if (tid == 0) gave_up = 0;
    fence_barrier_init();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int U = units_per_seq(a);
    const long long total = pages_before(c, c.B, scratch) * U;
    const int ctas = active_ctas(total);
    if ((int)blockIdx.x >= ctas) return;
    const long long cta0 = total * blockIdx.x / ctas, cta1 = total * (blockIdx.x + 1) / ctas;
    Cursor cur{0, 0, 0, 0};
    int remaining = 0;
    long long seg_at = 0;                              // index of the present segment's first page
    if (warp < W) {
        const long long nw = (long long)ctas * W, w0 = total * ((long long)blockIdx.x * W + warp) / nw;
        remaining = (int)(total * ((long long)blockIdx.x * W + warp + 1) / nw - w0);
        if (remaining > 0) cur = locate(c, U, w0, lane);
        seg_at = w0 - cur.p;
        if (lane == 0) {
            begin_of[warp] = cur;
            pages_of[warp] = remaining;
        }
    }
    __syncthreads();
    if (warp == W) {
        // ---- loads: lane i feeds consumer i, a half page at a time, whenever the consumer has read the one before
        if (lane < W) {
            Cursor ld = begin_of[lane];
            int halves = 2 * pages_of[lane], i = 0, id = halves ? c.page(ld.b, ld.p) : -1, kv = ld.u / a.blocks;
            const uint32_t dst = smem_u32(smem) + lane * C::PER_WARP, bar = smem_u32(smem) + C::BAR_OFF + 32 * lane;
            for (uint32_t polls = 0; i < halves && polls < (1u << 22); ++polls) {           // polls since the last load
                const int half = i & 1;
                // the first page finds its buffers empty; later ones wait for the reading of the page before
                if (i >= 2 && !mbar_test_wait(bar + 16 + 8 * half, (uint32_t)(i / 2 - 1) & 1u)) {
                    if ((polls & 63) == 63 && gave_up) break;
                    continue;
                }
                if (!half) page_there[lane] = id >= 0;             // read before V's half is released
                if (id >= 0) {
                    mbar_expect_tx(bar + 8 * half, P::HALF);
                    bulk_load(dst + half * P::HALF, c.pages + ((long long)id * c.Hkv + kv) * P::BYTES + half * P::HALF, P::HALF, bar + 8 * half);
                } else {
                    mbar_arrive(bar + 8 * half);                   // nothing to load: the tokens are left out
                }
                ++i;
                polls = 0;
                if (half && i < halves) {                          // the next page
                    if (++ld.p == ld.np) {
                        ld.p = 0;
                        if (++ld.u == U) {
                            ld.u = 0;
                            do { ++ld.b; } while ((ld.np = c.n_pages_of(ld.b)) == 0);
                        }
                        kv = ld.u / a.blocks;
                    }
                    id = c.page(ld.b, ld.p);
                }
            }
        }
        __syncwarp();
    }
    uint32_t phase = 0;
    bool ok = true;
#pragma unroll 1
    while (remaining > 0 && ok) {
        // ---- a segment: query operands
        const int kv = cur.u / a.blocks, len = c.len(cur.b);
        float f_log2[NT][2];                           // what makes a product a score times log2(e), columns 2t, 2t + 1
        int stat_row[NT][2];                           // (sequence, query head) of columns 2t, 2t + 1, -1: no such row
        int limit[NT][2];                              // keys that the rows of columns 2t, 2t + 1 see
        int full = len;                                // keys that every row sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int head = 0, tok = 0;
            const bool have = row_of<ROWS>(a, cur.u, nt * 8 + g, head, tok);
            const uint16_t* qp = (const uint16_t*)a.q + cur.b * a.qs.b + head * a.qs.h + tok * a.qs.t;
            uint32_t x[NG][8];                                      // elements 16t..16t+15 of each group
            float top = 0.f;
#pragma unroll
            for (int G = 0; G < NG; ++G) {
                uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                if (have) {
                    lo = __ldg(reinterpret_cast<const uint4*>(qp + 64 * G + 16 * t));
                    hi = __ldg(reinterpret_cast<const uint4*>(qp + 64 * G + 16 * t) + 1);
                }
                x[G][0] = lo.x; x[G][1] = lo.y; x[G][2] = lo.z; x[G][3] = lo.w;
                x[G][4] = hi.x; x[G][5] = hi.y; x[G][6] = hi.z; x[G][7] = hi.w;
                if (a.s) {                                          // FP32 product, rounded once to the activation dtype
                    const float4* sp = reinterpret_cast<const float4*>(a.s + kv * D + 64 * G + 16 * t);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 f = __ldg(sp + i);
                        float e0, e1;
                        Pair16<T>::unpack(x[G][2 * i], e0, e1);
                        x[G][2 * i] = Pair16<T>::round_pack(e0 * f.x, e1 * f.y);
                        Pair16<T>::unpack(x[G][2 * i + 1], e0, e1);
                        x[G][2 * i + 1] = Pair16<T>::round_pack(e0 * f.z, e1 * f.w);
                    }
                }
                if constexpr (BF) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float e0, e1;
                        Pair16<T>::unpack(x[G][i], e0, e1);
                        top = max3(top, fabsf(e0), fabsf(e1));
                    }
                }
            }
            // BF16 rows become FP16 rows times a power of two that brings their largest magnitude to [2^14, 2^15): exact down to
            // 2^-31 of it, and off by 2^-39 of it at most below
            float unscale = a.scale_log2;
            if constexpr (BF) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int E = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 127);
                const float up = __uint_as_float((uint32_t)(14 - E + 127) << 23);
                unscale = a.scale_log2 * __uint_as_float((uint32_t)(E - 14 + 127) << 23);
#pragma unroll
                for (int G = 0; G < NG; ++G)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float e0, e1;
                        Pair16<T>::unpack(x[G][i], e0, e1);
                        x[G][i] = Pair16<__half>::round_pack(e0 * up, e1 * up);
                    }
            }
            f_log2[nt][0] = __shfl_sync(0xffffffffu, unscale, 8 * t);       // of the rows of columns 2t, 2t + 1
            f_log2[nt][1] = __shfl_sync(0xffffffffu, unscale, 8 * t + 4);
#pragma unroll
            for (int G = 0; G < NG; ++G) {                          // pairs (i, i + 4) of each unit; a lane reads what it writes here
                const uint32_t at = qbuf + (nt * NG + G) * 1024;
                sts128(at, __byte_perm(x[G][0], x[G][2], 0x5410), __byte_perm(x[G][0], x[G][2], 0x7632),
                       __byte_perm(x[G][1], x[G][3], 0x5410), __byte_perm(x[G][1], x[G][3], 0x7632));
                sts128(at + 512, __byte_perm(x[G][4], x[G][6], 0x5410), __byte_perm(x[G][4], x[G][6], 0x7632),
                       __byte_perm(x[G][5], x[G][7], 0x5410), __byte_perm(x[G][5], x[G][7], 0x7632));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool row = row_of<ROWS>(a, cur.u, nt * 8 + 2 * t + e, head, tok);
                stat_row[nt][e] = row ? cur.b * a.Hq + head : -1;
                limit[nt][e] = len;
                if (a.causal && row) {
                    limit[nt][e] = len - a.N + 1 + tok;
                    full = min(full, limit[nt][e]);
                }
            }
        }
        if (a.causal) {
            full = min(full, __shfl_xor_sync(0xffffffffu, full, 1));
            full = min(full, __shfl_xor_sync(0xffffffffu, full, 2));
        }
        float o[D / 16][NT][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][nt][e] = 0.f;
        }
        const int first_p = cur.p, n_here = min(cur.np - cur.p, remaining);
#pragma unroll 1
        for (int pi = 0; pi < n_here; ++pi) {
            const int p = first_p + pi;
            // ---- S = K q~
            if (!__all_sync(0xffffffffu, mbar_wait(bars, phase))) { ok = false; break; }
            const bool there = page_there[warp];
            float s[4][NT][4];
            uint32_t qf[NT][NG][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int G = 0; G < NG; ++G)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint4 v = lds128(qbuf + (nt * NG + G) * 1024 + 512 * x);
                        qf[nt][G][x][0] = v.x; qf[nt][G][x][1] = v.y; qf[nt][G][x][2] = v.z; qf[nt][G][x][3] = v.w;
                    }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[2][NG][2], shw[2][NG];
                float sc[2][NG];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = 16 * i + 8 * r + g;
                    const uint32_t wa = kb + P::K_CODES + row * (D / 2) + t * 8 * NG;
                    if constexpr (NG == 1) {
                        const uint2 x = lds64(wa);
                        w[r][0][0] = x.x; w[r][0][1] = x.y;
                    } else {
#pragma unroll
                        for (int G = 0; G < NG; G += 2) {
                            const uint4 x = lds128(wa + 8 * G);
                            w[r][G][0] = x.x; w[r][G][1] = x.y; w[r][G + 1][0] = x.z; w[r][G + 1][1] = x.w;
                        }
                    }
#pragma unroll
                    for (int G = 0; G < NG; ++G) {
                        shw[r][G] = lds32(kb + P::K_SHIFTS + 4 * (row * NG + G));
                        sc[r][G] = half_scale(lds8(kb + P::K_SCALES + row * NG + G));
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][nt][e] = 0.f;
#pragma unroll
                for (int G = 0; G < NG; ++G) {
                    uint32_t A[2][2][4];                              // [row half][unit][step]
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t y = turn(shw[r][G], t);
                        unpack8(w[r][G][0], y, a.one, A[r][0]);
                        unpack8(w[r][G][1], y >> 2, a.one, A[r][1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma16816(acc, A[0][0][x], A[1][0][x], A[0][1][x], A[1][1][x], qf[nt][G][0][x], qf[nt][G][1][x]);
                        s[i][nt][0] = fmaf(acc[0], sc[0][G], s[i][nt][0]);
                        s[i][nt][1] = fmaf(acc[1], sc[0][G], s[i][nt][1]);
                        s[i][nt][2] = fmaf(acc[2], sc[1][G], s[i][nt][2]);
                        s[i][nt][3] = fmaf(acc[3], sc[1][G], s[i][nt][3]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 16);
            // ---- softmax of the page's tokens; lane: rows 16 i + g and 16 i + 8 + g, columns 2 t and 2 t + 1
            if (64 * p + 64 > full || !there) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!there || 64 * p + 16 * i + 8 * (e >> 1) + g >= limit[nt][e & 1]) s[i][nt][e] = -INFINITY;
            }
            bool moved = false;
            float f[NT][2];
            uint32_t pw[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = max3(mx, s[i][nt][e], s[i][nt][e + 2]);
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                    // the reference lies 15 below the maximum, so that P <= 2^15 fills the range of FP16
                    const float mn = fmaxf(m[nt][e], fmaf(mx, f_log2[nt][e], -15.f));
                    const float ref = mn == -INFINITY ? 0.f : mn;
                    f[nt][e] = ex2_approx(m[nt][e] - ref);
                    moved |= mn != m[nt][e];
                    m[nt][e] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = ex2_approx(fmaf(s[i][nt][e], f_log2[nt][e], -ref));
                        const float p1 = ex2_approx(fmaf(s[i][nt][e + 2], f_log2[nt][e], -ref));
                        sum += p0 + p1;
                        pw[nt][e][i] = Pair16<__half>::round_pack(p0, p1);
                    }
                    l[nt][e] = fmaf(l[nt][e], f[nt][e], sum);
                    if (a.page_ml) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                        if (g == 0 && stat_row[nt][e] >= 0) a.page_ml[(long long)stat_row[nt][e] * c.max_pages + p] = make_float2(mn, sum);
                    }
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[j][nt][e] *= f[nt][e & 1];
            }
            // ---- P as the second operand: word (i, g) of a column holds the tokens 16 i + g and 16 i + 8 + g
            uint32_t pf[NT][8];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sts32(pbuf + 4 * (nt * 8 * C::PV_ROW + (2 * t + e) * C::PV_ROW + 8 * i + g), pw[nt][e][i]);
            }
            __syncwarp();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint32_t pa = pbuf + 4 * (nt * 8 * C::PV_ROW + g * C::PV_ROW + 8 * t);
                const uint4 lo = lds128(pa), hi = lds128(pa + 16);
                pf[nt][0] = lo.x; pf[nt][1] = lo.y; pf[nt][2] = lo.z; pf[nt][3] = lo.w;
                pf[nt][4] = hi.x; pf[nt][5] = hi.y; pf[nt][6] = hi.z; pf[nt][7] = hi.w;
            }
            // ---- O += V^T P
            if (!__all_sync(0xffffffffu, mbar_wait(bars + 8, phase))) { ok = false; break; }
            if (there) {
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    uint32_t A[2][2][4];
                    float sc[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int ch = 16 * j + 8 * r + g;
                        const uint2 w = lds64(vb + P::K_CODES + ch * 32 + t * 8);
                        const uint32_t y = turn(lds32(vb + P::K_SHIFTS + 4 * ch), t);
                        sc[r] = half_scale(lds8(vb + P::K_SCALES + ch));
                        unpack8(w.x, y, a.one, A[r][0]);
                        unpack8(w.y, y >> 2, a.one, A[r][1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma16816(acc, A[0][0][x], A[1][0][x], A[0][1][x], A[1][1][x], pf[nt][x], pf[nt][4 + x]);
                        o[j][nt][0] = fmaf(acc[0], sc[0], o[j][nt][0]);
                        o[j][nt][1] = fmaf(acc[1], sc[0], o[j][nt][1]);
                        o[j][nt][2] = fmaf(acc[2], sc[1], o[j][nt][2]);
                        o[j][nt][3] = fmaf(acc[3], sc[1], o[j][nt][3]);
                    }
                }
            } else if (lane == 0) {
                c.invalid();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 24);
            phase ^= 1;
        }
        if (!ok) break;
        // ---- the segment's part is complete
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], x);
        remaining -= n_here;
        const bool begins = first_p == 0, ends = first_p + n_here == cur.np;
        if (begins && ends) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    int head, tok;
                    if (!row_of<ROWS>(a, cur.u, nt * 8 + 2 * t + e, head, tok)) continue;
                    const float inv = l[nt][e] == 0.f ? 0.f : 1.f / l[nt][e];
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        store_out(a, cur.b, head, tok, D, 16 * j + g, o[j][nt][e] * inv);
                        store_out(a, cur.b, head, tok, D, 16 * j + 8 + g, o[j][nt][e + 2] * inv);
                    }
                    if (g == 0) store_row_stats(a, cur.b, head, tok, m[nt][e], l[nt][e]);
                }
        } else {
            const int slot = begins ? 1 : 0;
            // the last piece goes where the page was; one that others follow, to global memory
            float* po = remaining == 0 ? reinterpret_cast<float*>(smem + warp * C::PER_WARP)
                                       : a.first + ((long long)blockIdx.x * W + warp) * C::PIECE;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = nt * 8 + 2 * t + e;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        po[r * D + 16 * j + g] = o[j][nt][e];
                        po[r * D + 16 * j + 8 + g] = o[j][nt][e + 2];
                    }
                    if (g == 0) {
                        po[ROWS * D + 2 * r] = m[nt][e];
                        po[ROWS * D + 2 * r + 1] = l[nt][e];
                    }
                }
            if (lane == 0) {
                piece[2 * warp + slot] = cur;
                piece_at[2 * warp + slot] = seg_at;
                piece_of[2 * warp + slot] = po;
            }
        }
        // next segment
        seg_at += cur.np;
        cur.p = 0;
        if (ends && remaining > 0) {
            if (++cur.u == U) {
                cur.u = 0;
                do { ++cur.b; } while (cur.b < c.B && (cur.np = c.n_pages_of(cur.b)) == 0);
            }
        }
    }
    if (!ok) {
        gave_up = 1;
        if (lane == 0 && c.d_status) *c.d_status = HIFA4_ERR_TIMEOUT;
        let_copies_land();
    }
    // ---- pieces that warps share: a (segment, row) per warp and turn
    __syncthreads();
    {
        const long long at = lane < 2 * W ? piece_at[lane] : -1;
        const unsigned first = __ballot_sync(0xffffffffu, !(lane & 1) && at >= 0 && at < cta0);   // of the segment that the CTA before began
        unsigned leaders = __ballot_sync(0xffffffffu, (lane & 1) && at >= 0) | (first & (0u - first));
        int unit = 0;
        while (leaders) {
            const int lead = __ffs(leaders) - 1;
            leaders &= leaders - 1;
            const long long seg = __shfl_sync(0xffffffffu, at, lead);
            const unsigned members = __ballot_sync(0xffffffffu, !(lane & 1) && at == seg) | (1u << lead);
            const Cursor sg = piece[lead];
            const bool whole = seg >= cta0 && seg + sg.np <= cta1;
            const int ws = 2 * (int)blockIdx.x + (seg < cta0 ? 0 : 1);
            const bool mine = members >> lane & 1;
            const float* const po = mine ? piece_of[lane] : nullptr;
#pragma unroll 1
            for (int r = 0; r < ROWS; ++r) {
                int head, tok;
                if (!row_of<ROWS>(a, sg.u, r, head, tok)) break;
                if (unit++ % (W + 1) != warp) continue;
                const float m = mine ? po[ROWS * D + 2 * r] : -INFINITY;
                const float M = warp_max(m), f = rebase(m, M);
                const float L = warp_sum(mine ? po[ROWS * D + 2 * r + 1] * f : 0.f);
                float o[D / 32];
#pragma unroll
                for (int x = 0; x < D / 32; ++x) o[x] = 0.f;
                for (unsigned rest = members; rest; rest &= rest - 1) {
                    const int x = __ffs(rest) - 1;
                    const float fx = __shfl_sync(0xffffffffu, f, x);
                    const float* px = piece_of[x] + r * D + lane;
#pragma unroll
                    for (int y = 0; y < D / 32; ++y) o[y] = fmaf(px[32 * y], fx, o[y]);
                }
                if (whole) {
                    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
                    for (int y = 0; y < D / 32; ++y) store_out(a, sg.b, head, tok, D, 32 * y + lane, o[y] * inv);
                    if (lane == 0) store_row_stats(a, sg.b, head, tok, M, L);
                } else {
                    float* dst = a.part_o + ((long long)ws * ROWS + r) * D + lane;
#pragma unroll
                    for (int y = 0; y < D / 32; ++y) dst[32 * y] = o[y];
                    if (lane == 0) a.part_ml[(long long)ws * ROWS + r] = make_float2(M, L);
                }
            }
        }
    }
}

// CTAs [0, DECODE_CTAS): the segment that begins in the CTA of this number and goes on in others, joined from their partial sums (a
// group of JOIN_WARPS / 8 warps per row, eight rows at a time), and the sequences without keys.  The rest: page weights, 64
// pages of a sequence each: sum over the query heads of (sum of p in the page) / (sum of p in all pages).
constexpr int JOIN_WARPS = 16;
template <int D, int ROWS>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
cache_join_kernel(const __grid_constant__ DecodeArgs a)
{
    constexpr int GROUP = JOIN_WARPS / 8;
    __shared__ long long scratch[JOIN_WARPS];
    __shared__ float part[JOIN_WARPS][D];
    __shared__ float2 ml_of[HIFA4_MAX_HEADS];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int U = units_per_seq(a), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long total = pages_before(c, c.B, scratch) * U;
    const int ctas = active_ctas(total);
    if (blockIdx.x >= DECODE_CTAS) {
        const int chunks = (c.max_pages + 63) / 64, w = (int)blockIdx.x - DECODE_CTAS, b = w / chunks, p0 = w % chunks * 64;
        const int np = c.n_pages_of(b);
        if (p0 >= np) return;
        const long long before = pages_before(c, b, scratch) * U;
        for (int j = tid; j < a.Hq; j += JOIN_WARPS * 32) {          // j: place among the query heads sorted by KV head
            int kv = 0;
            while (a.units.first[kv + 1] <= j) ++kv;
            const int in = j - a.units.first[kv], head = a.units.head[j], r = in % ROWS;
            const long long at = before + (long long)(kv * a.blocks + in / ROWS) * np;
            const long long c0 = ((at + 1) * ctas - 1) / total, c1 = ((at + np) * ctas - 1) / total;
            float2 ml;
            if (c0 == c1) {
                ml = a.final_ml[(long long)b * a.Hq + head];
            } else {
                ml = make_float2(-INFINITY, 0.f);
                for (long long x = c0; x <= c1; ++x) ml.x = fmaxf(ml.x, a.part_ml[(2 * x + (x == c0)) * ROWS + r].x);
                for (long long x = c0; x <= c1; ++x) {
                    const float2 y = a.part_ml[(2 * x + (x == c0)) * ROWS + r];
                    ml.y = fmaf(y.y, rebase(y.x, ml.x), ml.y);
                }
            }
            ml_of[head] = make_float2(ml.x, ml.y == 0.f ? 0.f : 1.f / ml.y);
        }
        __syncthreads();
        const int p = p0 + (tid & 63), grp = tid >> 6;
        constexpr int GROUPS = JOIN_WARPS / 2;
        float w_sum = 0.f;
        if (p < np) {
            const float2* src = a.page_ml + (long long)b * a.Hq * c.max_pages + p;
#pragma unroll 4
            for (int h = grp; h < a.Hq; h += GROUPS) {
                const float2 ml = src[(long long)h * c.max_pages], all = ml_of[h];
                w_sum = fmaf(ml.y * rebase(ml.x, all.x), all.y, w_sum);
            }
        }
        float* sums = &part[0][0];
        sums[tid] = w_sum;
        __syncthreads();
        if (grp == 0 && p < np) {
#pragma unroll
            for (int i = 1; i < GROUPS; ++i) w_sum += sums[64 * i + tid];
            const long long i = (long long)b * c.max_pages + p;
            a.weight_out[i] = (a.weight ? a.weight[i] : 0.f) + w_sum;
        }
        return;
    }
    for (int b = blockIdx.x; b < c.B; b += DECODE_CTAS) {            // no keys: zeros
        if (c.n_pages_of(b) > 0) continue;
        if (tid == 0 && c.len(b) < 0) c.invalid();
        for (int i = tid; i < a.Hq * a.N * D; i += JOIN_WARPS * 32) {
            const int head = i / (a.N * D), tok = i / D % a.N;
            store_out(a, b, head, tok, D, i % D, 0.f);
            if (i % D == 0) store_row_stats(a, b, head, tok, -INFINITY, 0.f);
        }
    }
    if ((int)blockIdx.x + 1 >= ctas) return;                          // nothing goes on behind the last CTA
    const long long cta0 = total * blockIdx.x / ctas, cta1 = total * (blockIdx.x + 1) / ctas;
    const Cursor sg = locate(c, U, cta1 - 1, lane);
    const long long at = cta1 - 1 - sg.p;
    if (at < cta0 || at + sg.np == cta1) return;
    const int c0 = blockIdx.x, n = (int)(((at + sg.np) * ctas - 1) / total) - c0 + 1;
    const int per = (n + GROUP - 1) / GROUP, x0 = min(n, warp % GROUP * per), x1 = min(n, x0 + per);
    auto slot_of = [&](int x) { return (long long)(2 * (c0 + x) + (x == 0 ? 1 : 0)) * ROWS; };
#pragma unroll 1
    for (int r0 = 0; r0 < ROWS; r0 += 8) {
        const int r = r0 + warp / GROUP;
        int head, tok;
        const bool have = row_of<ROWS>(a, sg.u, r, head, tok);
        float M = -INFINITY, L = 0.f, o[D / 32];
#pragma unroll
        for (int y = 0; y < D / 32; ++y) o[y] = 0.f;
        if (have) {
            for (int x = lane; x < n; x += 32) M = fmaxf(M, a.part_ml[slot_of(x) + r].x);
            M = warp_max(M);
            for (int x = lane; x < n; x += 32) {
                const float2 ml = a.part_ml[slot_of(x) + r];
                L = fmaf(ml.y, rebase(ml.x, M), L);
            }
            L = warp_sum(L);
#pragma unroll 8
            for (int x = x0; x < x1; ++x) {
                const float f = rebase(a.part_ml[slot_of(x) + r].x, M);
                const float* src = a.part_o + (slot_of(x) + r) * D + lane;
#pragma unroll
                for (int y = 0; y < D / 32; ++y) o[y] = fmaf(src[32 * y], f, o[y]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < D / 32; ++y) part[warp][32 * y + lane] = o[y];
        __syncthreads();
        if (have && warp % GROUP == 0) {
            const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
            for (int y = 0; y < D / 32; ++y) {
#pragma unroll
                for (int x = 1; x < GROUP; ++x) o[y] += part[warp + x][32 * y + lane];
                store_out(a, sg.b, head, tok, D, 32 * y + lane, o[y] * inv);
            }
            if (lane == 0) store_row_stats(a, sg.b, head, tok, M, L);
        }
    }
}

int decode_block_rows(int d, int rows) { return rows <= 8 || d == 256 ? 8 : 16; }

size_t decode_first_floats(int d, int block_rows) { return (size_t)DECODE_CTAS * 16 * block_rows * (d + 2); }

template <typename T, int D, int NT>
static cudaError_t decode_nt(const DecodeArgs& a, cudaStream_t st)
{
    using C = DecodeCfg<D, NT>;
    static SmemOptIn opt;
    if (!opt.ensure(cache_decode_kernel<T, D, NT>, C::SMEM)) return cudaErrorInvalidValue;
    const cudaError_t e = launch_dependent(cache_decode_kernel<T, D, NT>, DECODE_CTAS, C::THREADS, C::SMEM, st, a);
    if (e != cudaSuccess) return e;
    const unsigned weight_blocks = a.weight_out ? (unsigned)a.cache.B * ((unsigned)(a.cache.max_pages + 63) / 64) : 0;
    return launch_dependent(cache_join_kernel<D, C::ROWS>, DECODE_CTAS + weight_blocks, JOIN_WARPS * 32, 0, st, a);
}

template <typename T>
static cudaError_t decode_t(int d, int block_rows, const DecodeArgs& a, cudaStream_t st)
{
    switch (d * 100 + block_rows) {
    case 6408: return decode_nt<T, 64, 1>(a, st);
    case 6416: return decode_nt<T, 64, 2>(a, st);
    case 12808: return decode_nt<T, 128, 1>(a, st);
    case 12816: return decode_nt<T, 128, 2>(a, st);
    default: return decode_nt<T, 256, 1>(a, st);
    }
}

cudaError_t launch_cache_decode(int dtype, int d, int block_rows, const DecodeArgs& a, cudaStream_t st)
{
    return dtype == HIFA4_BF16 ? decode_t<__nv_bfloat16>(d, block_rows, a, st) : decode_t<__half>(d, block_rows, a, st);
}

}  // namespace hifa4
