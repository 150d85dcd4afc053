// Attention of a few query rows per KV head over the paged HIF4 cache, split over the caches' lengths and joined.
//
//   S = q~ K^T scale,  m = running max,  p = exp2(S log2e - m + 15),  l = sum p,  O = p V / l
//
// Work: the (sequence, block of query rows of a KV head, page) triples of all sequences, in this order, are dealt out to the
// consumer warps of one CTA per SM in contiguous ranges of equal cost, whatever the sequences' lengths: a page costs two steps,
// beginning a (sequence, block) one (400 of 1500 instructions, and what it stores).  A consumer takes whole pages on
// its own: it forms S of the page's 64 tokens, its softmax and O, all in registers, without any exchange between
// warps.  At d = 256, where registers leave room for 7 such warps only, a consumer is a pair of warps: each forms S of half the
// page's tokens and O of half the channels; maxima and P pass through shared memory (8 sequences of 5-8K tokens, 16 / 8 heads:
// 54 us with single warps, 48.5 with pairs).  One more warp loads the pages (bulk copies, a lane per consumer).  The pages of one
// (sequence, block) that a range holds are a piece of its segment; pieces that consumers of one CTA share are joined in shared
// memory, those that CTAs share by a second, small kernel.
//
// Products run on mma.sync m16n8k16 with the cache as the 16-row operand, tokens (S) or channels (O) its rows, and query rows as the
// 8 columns: an operand of 5 or 6 query rows would leave a 128-row tcgen05 tile nearly empty, and its other operand would have to
// pass through shared memory as 16-bit values, four times the bytes of the codes.  Here codes become FP16 operands in
// registers (code * 2^shift, at most 28 in magnitude, exact); the scale of a group multiplies the FP32 sums of the
// group's products, per token for S, per channel for O.  Any order of the contraction index will do as long as both operands
// agree on it, so each lane takes whole 8-code words.
#include "hifa4_cache.cuh"

#include <algorithm>

namespace hifa4 {

using namespace ptx;

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same from zero (an operand that is a register set to zero first costs that instruction).
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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

// NT: 8-row column tiles of query rows.  A consumer (a warp, or a pair of them) has room for one page; the K half is loaded again
// while V is multiplied, and the other way round.  The query operands wait in shared memory while V is multiplied.
template <int D, int NT> struct DecodeCfg {
    static constexpr int W = D == 256 ? 7 : NT == 1 ? 15 : D == 128 ? 7 : 11;   // consumers
    static constexpr int PAIR = D == 256 ? 2 : 1;                        // warps of a consumer
    static constexpr int WARPS = W * PAIR + 1, THREADS = WARPS * 32;
    static constexpr int ROWS = 8 * NT;
    static constexpr int PV_ROW = 36;                                    // words of P per query row: 32 and 4 against bank conflicts
    static constexpr int PIECE = ROWS * (D + 2);                         // floats of a partial result: O [ROWS][D], then (m, l) [ROWS]
    static constexpr int K_OFF = 0, V_OFF = Page<D>::HALF, P_OFF = Page<D>::BYTES, Q_OFF = P_OFF + NT * 8 * PV_ROW * 4;
    static constexpr int PER_WARP = Q_OFF + PAIR * ROWS * D * 2;
    static constexpr int BAR_OFF = W * PER_WARP;                         // per consumer: K landed, V landed, K read, V read
    static constexpr int SMEM = BAR_OFF + W * 32 + 64;
    static_assert(PER_WARP % 16 == 0 && Page<D>::HALF % 16 == 0 && PIECE * 4 <= PER_WARP && SMEM <= 227 * 1024 - 2048, "shared memory");
};

// A position in the list of work: page `p` of `np` of unit `u` of sequence `b`.
struct Cursor {
    int b, u, p, np;
};

// Inclusive prefix sum over a warp.
__device__ __forceinline__ int warp_scan(int x, int lane)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// Steps of a (sequence, block) of np pages.  Page p is step 2 p + 1; a range of steps has the pages whose steps are in it.
__device__ __forceinline__ int steps_of(int np) { return np ? 2 * np + 1 : 0; }

// Steps of all sequences, for one block each.  Every warp sums for itself where that takes few loads (no barrier to wait for),
// else the block does.  All threads of the block call it together and get the sum.
__device__ __forceinline__ int all_steps(const CacheView& c, int* scratch)
{
    int s = 0;
    if (c.B <= 128) {
        for (int b = threadIdx.x & 31; b < c.B; b += 32) s += steps_of(c.n_pages_of(b));
        return __reduce_add_sync(0xffffffffu, s);
    }
    for (int b = threadIdx.x; b < c.B; b += blockDim.x) s += steps_of(c.n_pages_of(b));
    s = __reduce_add_sync(0xffffffffu, s);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    int t = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) t += scratch[w];
    return t;
}

// The first page at or behind step `at` of the list of work (at is less than the list's length; np = 0: there is none), its
// index among all pages and its segment's first step.  Whole warp.
__device__ __forceinline__ Cursor locate(const CacheView& c, int U, int at, int lane, int* index, int* seg)
{
    Cursor cur{0, 0, 0, 0};
    int steps = 0, pages = 0;                          // of the sequences before
    for (int b0 = 0; b0 < c.B; b0 += 32) {
        const int np = b0 + lane < c.B ? c.n_pages_of(b0 + lane) : 0, pre = warp_scan(steps_of(np), lane), pre_p = warp_scan(np, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, (steps + pre) * U > at);
        if (hit) {
            const int l = __ffs(hit) - 1;
            cur.b = b0 + l;
            cur.np = __shfl_sync(0xffffffffu, np, l);
            steps += __shfl_sync(0xffffffffu, pre - steps_of(np), l);
            pages += __shfl_sync(0xffffffffu, pre_p - np, l);
            break;
        }
        steps += __shfl_sync(0xffffffffu, pre, 31);
        pages += __shfl_sync(0xffffffffu, pre_p, 31);
    }
    const int in = at - steps * U, size = steps_of(cur.np);
    cur.u = (int)((unsigned)in / (unsigned)size);
    cur.p = (in - cur.u * size) >> 1;
    *seg = steps * U + cur.u * size;
    *index = pages * U + cur.u * cur.np + cur.p;
    if (cur.p == cur.np) {                             // the last step of a segment: on to the next one
        *seg += size;
        cur.p = 0;
        if (++cur.u == U) {
            cur.u = 0;
            do { ++cur.b; } while (cur.b < c.B && c.n_pages_of(cur.b) == 0);
            cur.np = cur.b < c.B ? c.n_pages_of(cur.b) : 0;
        }
    }
    return cur;
}

// Equal shares of n things for `parts`: where share i begins, the first n % parts being one longer; and whose thing x is.
struct Shares {
    int per, more;
    __device__ __forceinline__ Shares(int n, int parts) : per((int)((unsigned)n / (unsigned)parts)), more(n - per * parts) {}
    __device__ __forceinline__ int begin(int i) const { return i * per + min(i, more); }
    __device__ __forceinline__ int owner(int x) const
    {
        const int cut = more * (per + 1);
        return x < cut ? (int)((unsigned)x / (unsigned)(per + 1)) : more + (int)((unsigned)(x - cut) / (unsigned)per);
    }
};

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

// CTAs that take part: two steps each at least, so that every one that a segment passes through has a page of it.
__device__ __forceinline__ int active_ctas(int total) { return min(DECODE_CTAS, total / 2); }

__device__ __forceinline__ int units_per_seq(const DecodeArgs& a) { return a.cache.Hkv * a.blocks; }

__device__ __forceinline__ int kv_of(const DecodeArgs& a, int u) { return a.blocks == 1 ? u : (int)((unsigned)u / (unsigned)a.blocks); }

// Row r of unit u: query head and token; false behind the last row.
template <int ROWS>
__device__ __forceinline__ bool row_of(const DecodeArgs& a, int u, int r, int& head, int& tok)
{
    const int kv = kv_of(a, u), i = (u - kv * a.blocks) * ROWS + r;
    const int first = a.units.first[kv], n = (a.units.first[kv + 1] - first) * a.N;
    if (i >= n) return false;
    const int h = a.N == 1 ? i : (int)((unsigned)i / (unsigned)a.N);
    head = a.units.head[first + h];
    tok = i - h * a.N;
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

// A lane's share of the query rows of a segment, 16 channels of each group of row nt * 8 + g.
template <int D, int NT> struct QueryLoad {
    uint4 x[NT][D / 64][2];
    template <int ROWS> __device__ __forceinline__ void issue(const DecodeArgs& a, const Cursor& cur, int g, int t)
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int head = 0, tok = 0;
            const bool have = row_of<ROWS>(a, cur.u, nt * 8 + g, head, tok);
            const uint4* p = reinterpret_cast<const uint4*>((const uint16_t*)a.q + cur.b * a.qs.b + head * a.qs.h + tok * a.qs.t) + 2 * t;
#pragma unroll
            for (int G = 0; G < D / 64; ++G)
#pragma unroll
                for (int i = 0; i < 2; ++i) x[nt][G][i] = have ? __ldg(p + 8 * G + i) : make_uint4(0, 0, 0, 0);
        }
    }
};

// Factor that takes sums under the reference m to the reference M >= m (both -inf: nothing there).
__device__ __forceinline__ float rebase(float m, float M) { return m == -INFINITY ? 0.f : exp2f(m - M); }

// Both warps of consumer i meet (named barrier i + 1); whether x holds for both: neither waits for one that gave up.
__device__ __forceinline__ bool pair_sync(int i, bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x), "r"(i + 1) : "memory");
    return r != 0;
}

// SELFTEST (hifa4_selftest_cache_wait_timeout): in the first CTA the loader leaves out the first consumer's second page, and that
// consumer gives up on it after 2^6 polls.
template <typename T, int D, int NT, bool SELFTEST>
__global__ void __launch_bounds__(DecodeCfg<D, NT>::THREADS, 1)
cache_decode_kernel(const __grid_constant__ DecodeArgs a)
{
    using C = DecodeCfg<D, NT>;
    using P = Page<D>;
    constexpr int NG = P::NG, W = C::W, ROWS = C::ROWS, PAIR = C::PAIR;
    static_assert(PAIR == 1 || NT == 1, "a pair exchanges 8 rows");
    constexpr int TI = 4 / PAIR, CJ = D / 16 / PAIR;   // a warp's 16-token and 16-channel tiles of a page
    constexpr bool BF = sizeof(T) == 2 && !__is_same(T, __half);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int scratch[C::WARPS];
    __shared__ Cursor begin_of[W + 1];                 // first page of a consumer's range
    __shared__ int first_page[W + 1];                  // its index among all pages
    __shared__ volatile int now[W * PAIR][6];          // what a warp does not hold in registers while it goes through pages: the
                                                       // present segment (Cursor), its first step, the pages left
    __shared__ volatile int plan[4];                   // steps in all, CTAs, this CTA's first step and the one behind its last
    __shared__ volatile int page_there[W];             // whether the page in a consumer's buffers exists
    __shared__ volatile int gave_up;
    __shared__ Cursor piece[2 * W];                    // pieces of segments that a consumer shares with others: [2 w] begun before it,
                                                       // [2 w + 1] in it
    __shared__ int piece_at[2 * W];                    // the segment's first step, -1: no such piece
    __shared__ float* piece_of[2 * W];                 // where it is
    constexpr int PAIRS = PAIR == 2 ? W : 1;           // what the two warps of a consumer tell each other, per query row
    __shared__ volatile float pair_max[PAIRS][2][8], pair_sum[PAIRS][2][8], pair_l[PAIRS][2][8];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int cons = warp / PAIR, half = warp % PAIR;  // (the loader: consumer W)
    const uint32_t base = smem_u32(smem) + cons * C::PER_WARP;
    const uint32_t kb = base + C::K_OFF, vb = base + C::V_OFF, pbuf = base + C::P_OFF, qbuf = base + C::Q_OFF + half * ROWS * D * 2 + 16 * lane;
    const uint32_t bars = smem_u32(smem) + C::BAR_OFF + cons * 32;
    if (tid < 4 * W) mbar_init(smem_u32(smem) + C::BAR_OFF + 8 * tid, tid & 2 ? PAIR : 1);
    if (tid < 2 * W) piece_at[tid] = -1;
    if (tid == 0) gave_up = 0;
    fence_barrier_init();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int U = units_per_seq(a);
    const int total = all_steps(c, scratch) * U, ctas = active_ctas(total);
    if ((int)blockIdx.x >= ctas) {
        if (tid == 0) a.begun[blockIdx.x].x = -1;
        return;
    }
    const Shares of_ctas(total, ctas);
    const int cta0 = of_ctas.begin(blockIdx.x), cta1 = of_ctas.begin(blockIdx.x + 1);
    QueryLoad<D, NT> ql;
    {
        const Shares of_warps(cta1 - cta0, W);
        const int w0 = cta0 + of_warps.begin(cons);    // the loader: where the next CTA begins
        int index, seg_at;
        const Cursor cur = locate(c, U, min(w0, total - 1), lane, &index, &seg_at);
        if (cons < W && cur.np > 0) ql.template issue<ROWS>(a, cur, g, t);      // ahead of the flood of page loads
        if (lane == 0) {
            if (half == 0) {
                begin_of[cons] = cur;
                first_page[cons] = index;
            }
            if (cons < W) {
                now[warp][0] = cur.b; now[warp][1] = cur.u; now[warp][2] = cur.p; now[warp][3] = cur.np; now[warp][4] = seg_at;
            }
        }
        if (tid == 0) { plan[0] = total; plan[1] = ctas; plan[2] = cta0; plan[3] = cta1; }
    }
    __syncthreads();
    if (cons < W && lane == 0) now[warp][5] = first_page[cons + 1] - first_page[cons];
    __syncwarp();
    if (cons == W) {
        // ---- loads: lane i feeds consumer i, a half page at a time, whenever the consumer has read the one before
        if (lane < W) {
            Cursor ld = begin_of[lane];
            int halves = 2 * (first_page[lane + 1] - first_page[lane]), i = 0, id = halves ? c.page(ld.b, ld.p) : -1, kv = kv_of(a, ld.u);
            const uint32_t dst = smem_u32(smem) + lane * C::PER_WARP, bar = smem_u32(smem) + C::BAR_OFF + 32 * lane;
            for (uint32_t polls = 0; i < halves && polls < (1u << 20); ++polls) {           // polls since the last load
                if (SELFTEST && blockIdx.x == 0 && lane == 0 && i == 2) break;
                const int half = i & 1;
                // the first page finds its buffers empty; later ones wait for the reading of the page before
                if (i >= 2 && !mbar_test_wait(bar + 16 + 8 * half, (uint32_t)(i / 2 - 1) & 1u)) {
                    if ((polls & 63) == 63 && gave_up) break;
                    __nanosleep(100);                              // half a page takes 2 us: no hurry, and polls take issue slots
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
                        kv = kv_of(a, ld.u);
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
    while (cons < W && now[warp][5] > 0) {
        // ---- a segment: query operands
        Cursor cur{now[warp][0], now[warp][1], now[warp][2], now[warp][3]};
        const int kv = kv_of(a, cur.u), len = c.len(cur.b);
        float f_log2[NT][2];                           // what makes a product a score times log2(e), columns 2t, 2t + 1
        int stat_row[NT][2];                           // (sequence, query head) of columns 2t, 2t + 1, -1: no such row
        int limit[NT][2];                              // keys that the rows of columns 2t, 2t + 1 see
        int full = len;                                // keys that every row sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int head = 0, tok = 0;
            uint32_t x[NG][8];                                      // elements 16t..16t+15 of each group
            float top = 0.f;
#pragma unroll
            for (int G = 0; G < NG; ++G) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 v = ql.x[nt][G][i];
                    x[G][4 * i] = v.x; x[G][4 * i + 1] = v.y; x[G][4 * i + 2] = v.z; x[G][4 * i + 3] = v.w;
                }
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
        float o[CJ][NT][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int j = 0; j < CJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][nt][e] = 0.f;
        }
        const int end_p = min(cur.np, cur.p + now[warp][5]);
#pragma unroll 1
        for (int p = cur.p; p < end_p; ++p) {
            // ---- S = K q~
            const bool k_in = __all_sync(0xffffffffu, mbar_wait(bars, phase, SELFTEST && blockIdx.x == 0 && cons == 0 && phase ? 1u << 6 : 1u << 18));
            if (PAIR == 1 && !k_in) { ok = false; break; }
            const bool there = page_there[cons];
            float s[TI][NT][4];
            constexpr int GS = NG < 2 ? NG : 2;                       // groups at a time
#pragma unroll
            for (int G0 = 0; G0 < NG; G0 += GS) {
                uint32_t qf[NT][GS][2][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int G = 0; G < GS; ++G)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint4 v = lds128(qbuf + (nt * NG + G0 + G) * 1024 + 512 * x);
                            qf[nt][G][x][0] = v.x; qf[nt][G][x][1] = v.y; qf[nt][G][x][2] = v.z; qf[nt][G][x][3] = v.w;
                        }
#pragma unroll
                for (int i = 0; i < TI; ++i) {
                    uint32_t w[2][GS][2], shw[2][GS];
                    float sc[2][GS];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int row = 16 * (TI * half + i) + 8 * r + g;
                        const uint32_t wa = kb + P::K_CODES + row * (D / 2) + t * 8 * NG + 8 * G0;
                        if constexpr (GS == 1) {
                            const uint2 x = lds64(wa);
                            w[r][0][0] = x.x; w[r][0][1] = x.y;
                        } else {
                            const uint4 x = lds128(wa);
                            w[r][0][0] = x.x; w[r][0][1] = x.y; w[r][1][0] = x.z; w[r][1][1] = x.w;
                        }
#pragma unroll
                        for (int G = 0; G < GS; ++G) {
                            shw[r][G] = lds32(kb + P::K_SHIFTS + 4 * (row * NG + G0 + G));
                            sc[r][G] = half_scale(lds8(kb + P::K_SCALES + row * NG + G0 + G));
                        }
                    }
#pragma unroll
                    for (int G = 0; G < GS; ++G) {
                        uint32_t A[2][2][4];                              // [row half][unit][step]
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const uint32_t y = turn(shw[r][G], t);
                            unpack8(w[r][G][0], y, a.one, A[r][0]);
                            unpack8(w[r][G][1], y >> 2, a.one, A[r][1]);
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float acc[4];
                            mma16816_first(acc, A[0][0][0], A[1][0][0], A[0][1][0], A[1][1][0], qf[nt][G][0][0], qf[nt][G][1][0]);
#pragma unroll
                            for (int x = 1; x < 4; ++x)
                                mma16816(acc, A[0][0][x], A[1][0][x], A[0][1][x], A[1][1][x], qf[nt][G][0][x], qf[nt][G][1][x]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[i][nt][e] = G0 + G ? fmaf(acc[e], sc[e >> 1][G], s[i][nt][e]) : acc[e] * sc[e >> 1][G];
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 16);
            // ---- softmax of the page's tokens; lane: rows 16 i + g and 16 i + 8 + g, columns 2 t and 2 t + 1
            if (64 * p + 64 > full || !there) {
#pragma unroll
                for (int i = 0; i < TI; ++i)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!there || 64 * p + 16 * (TI * half + i) + 8 * (e >> 1) + g >= limit[nt][e & 1]) s[i][nt][e] = -INFINITY;
            }
            bool moved = false;
            float f[NT][2], mx[NT][2];
            uint32_t pw[NT][2][TI];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    mx[nt][e] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < TI; ++i) mx[nt][e] = max3(mx[nt][e], s[i][nt][e], s[i][nt][e + 2]);
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) mx[nt][e] = fmaxf(mx[nt][e], __shfl_xor_sync(0xffffffffu, mx[nt][e], x));
                }
            if constexpr (PAIR == 2) {
                if (g == 0) { pair_max[cons][half][2 * t] = mx[0][0]; pair_max[cons][half][2 * t + 1] = mx[0][1]; }
                if (!pair_sync(cons, k_in)) { ok = false; break; }
#pragma unroll
                for (int e = 0; e < 2; ++e) mx[0][e] = fmaxf(mx[0][e], pair_max[cons][half ^ 1][2 * t + e]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // the reference lies 15 below the maximum, so that P <= 2^15 fills the range of FP16
                    const float mn = fmaxf(m[nt][e], fmaf(mx[nt][e], f_log2[nt][e], -15.f));
                    const float ref = mn == -INFINITY ? 0.f : mn;
                    f[nt][e] = ex2_approx(m[nt][e] - ref);
                    moved |= mn != m[nt][e];
                    m[nt][e] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < TI; ++i) {
                        const float p0 = ex2_approx(fmaf(s[i][nt][e], f_log2[nt][e], -ref));
                        const float p1 = ex2_approx(fmaf(s[i][nt][e + 2], f_log2[nt][e], -ref));
                        sum += p0 + p1;
                        pw[nt][e][i] = Pair16<__half>::round_pack(p0, p1);
                    }
                    l[nt][e] = fmaf(l[nt][e], f[nt][e], sum);
                    if (a.page_ml) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                        if (PAIR == 2 && g == 0) pair_sum[cons][half][2 * t + e] = sum;
                        if (PAIR == 1 && g == 0 && stat_row[nt][e] >= 0) a.page_ml[(long long)stat_row[nt][e] * c.max_pages + p] = make_float2(mn, sum);
                    }
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int j = 0; j < CJ; ++j)
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
                    for (int i = 0; i < TI; ++i) sts32(pbuf + 4 * (nt * 8 * C::PV_ROW + (2 * t + e) * C::PV_ROW + 8 * (TI * half + i) + g), pw[nt][e][i]);
            }
            const bool v_in = PAIR == 1 || __all_sync(0xffffffffu, mbar_wait(bars + 8, phase));
            if constexpr (PAIR == 1) {
                __syncwarp();
            } else {
                if (!pair_sync(cons, v_in)) { ok = false; break; }
                if (a.page_ml && half == 0 && g == 0)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (stat_row[0][e] >= 0)
                            a.page_ml[(long long)stat_row[0][e] * c.max_pages + p] =
                                make_float2(m[0][e], pair_sum[cons][0][2 * t + e] + pair_sum[cons][1][2 * t + e]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint32_t pa = pbuf + 4 * (nt * 8 * C::PV_ROW + g * C::PV_ROW + 8 * t);
                const uint4 lo = lds128(pa), hi = lds128(pa + 16);
                pf[nt][0] = lo.x; pf[nt][1] = lo.y; pf[nt][2] = lo.z; pf[nt][3] = lo.w;
                pf[nt][4] = hi.x; pf[nt][5] = hi.y; pf[nt][6] = hi.z; pf[nt][7] = hi.w;
            }
            // ---- O += V^T P
            if (PAIR == 1 && !__all_sync(0xffffffffu, mbar_wait(bars + 8, phase))) { ok = false; break; }
            if (there) {
#pragma unroll
                for (int j = 0; j < CJ; ++j) {
                    uint32_t A[2][2][4];
                    float sc[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int ch = 16 * (CJ * half + j) + 8 * r + g;
                        const uint2 w = lds64(vb + P::K_CODES + ch * 32 + t * 8);
                        const uint32_t y = turn(lds32(vb + P::K_SHIFTS + 4 * ch), t);
                        sc[r] = half_scale(lds8(vb + P::K_SCALES + ch));
                        unpack8(w.x, y, a.one, A[r][0]);
                        unpack8(w.y, y >> 2, a.one, A[r][1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float acc[4];
                        mma16816_first(acc, A[0][0][0], A[1][0][0], A[0][1][0], A[1][1][0], pf[nt][0], pf[nt][4]);
#pragma unroll
                        for (int x = 1; x < 4; ++x)
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
        if constexpr (PAIR == 2) {                                   // (and both have read their last page)
            if (g == 0) { pair_l[cons][half][2 * t] = l[0][0]; pair_l[cons][half][2 * t + 1] = l[0][1]; }
            pair_sync(cons, true);
#pragma unroll
            for (int e = 0; e < 2; ++e) l[0][e] = pair_l[cons][0][2 * t + e] + pair_l[cons][1][2 * t + e];
        }
        cur = Cursor{now[warp][0], now[warp][1], now[warp][2], now[warp][3]};
        const int seg_at = now[warp][4], remaining = now[warp][5] - (end_p - cur.p);
        const bool begins = cur.p == 0, ends = end_p == cur.np;
        if (begins && a.seg_ctas && half == 0 && lane == 0)                      // for the page weights: the CTAs that hold the segment
            a.seg_ctas[(long long)cur.b * units_per_seq(a) + cur.u] = make_int2(blockIdx.x, Shares(plan[0], plan[1]).owner(seg_at + 2 * cur.np - 1));
        if (begins && ends) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    int head, tok;
                    if (!row_of<ROWS>(a, cur.u, nt * 8 + 2 * t + e, head, tok)) continue;
                    const float inv = l[nt][e] == 0.f ? 0.f : 1.f / l[nt][e];
#pragma unroll
                    for (int j = 0; j < CJ; ++j) {
                        store_out(a, cur.b, head, tok, D, 16 * (CJ * half + j) + g, o[j][nt][e] * inv);
                        store_out(a, cur.b, head, tok, D, 16 * (CJ * half + j) + 8 + g, o[j][nt][e + 2] * inv);
                    }
                    if (half == 0 && g == 0) store_row_stats(a, cur.b, head, tok, m[nt][e], l[nt][e]);
                }
        } else {
            const int slot = begins ? 1 : 0;
            // the last piece goes where the page was; one that others follow, to global memory
            float* po = remaining == 0 ? reinterpret_cast<float*>(smem + cons * C::PER_WARP)
                                       : a.first + ((long long)blockIdx.x * W + cons) * C::PIECE;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = nt * 8 + 2 * t + e;
#pragma unroll
                    for (int j = 0; j < CJ; ++j) {
                        po[r * D + 16 * (CJ * half + j) + g] = o[j][nt][e];
                        po[r * D + 16 * (CJ * half + j) + 8 + g] = o[j][nt][e + 2];
                    }
                    if (half == 0 && g == 0) {
                        po[ROWS * D + 2 * r] = m[nt][e];
                        po[ROWS * D + 2 * r + 1] = l[nt][e];
                    }
                }
            if (half == 0 && lane == 0) {
                piece[2 * cons + slot] = cur;
                piece_at[2 * cons + slot] = seg_at;
                piece_of[2 * cons + slot] = po;
            }
        }
        // next segment
        const int next_at = seg_at + steps_of(cur.np);
        cur.p = 0;
        if (ends && remaining > 0) {
            const int U = units_per_seq(a);
            if (++cur.u == U) {
                cur.u = 0;
                do { ++cur.b; } while (cur.b < c.B && (cur.np = c.n_pages_of(cur.b)) == 0);
            }
            ql.template issue<ROWS>(a, cur, g, t);
        }
        __syncwarp();                                               // (every lane has read)
        if (lane == 0) {
            now[warp][0] = cur.b; now[warp][1] = cur.u; now[warp][2] = 0; now[warp][3] = cur.np; now[warp][4] = next_at; now[warp][5] = remaining;
        }
        __syncwarp();
    }
    if (!ok) {
        gave_up = 1;
        if (lane == 0) c.timed_out();
        let_copies_land();
    }
    // ---- pieces that warps share: a row of a segment per warp and turn
    __syncthreads();
    const int at = lane < 2 * W ? piece_at[lane] : -1, cta_first = plan[2], cta_end = plan[3];
    const bool second = lane & 1;
    const unsigned first = __ballot_sync(0xffffffffu, !second && at >= 0 && at + 1 < cta_first);      // of the segment that a CTA before began
    unsigned leaders = __ballot_sync(0xffffffffu, second && at >= 0) | (first & (0u - first));
    const unsigned cross = __ballot_sync(0xffffffffu, second && at >= 0 && at + 2 * piece[lane].np - 1 >= cta_end);
    if (tid == 0) {                                                  // what the join finds here
        int4 x = make_int4(-1, 0, 0, 0);
        if (cross) {
            const Cursor sg = piece[__ffs(cross) - 1];
            x = make_int4(sg.b, sg.u, Shares(plan[0], plan[1]).owner(piece_at[__ffs(cross) - 1] + 2 * sg.np - 1), 0);
        }
        a.begun[blockIdx.x] = x;
    }
    int turn = warp;
    while (leaders) {
        const int lead = __ffs(leaders) - 1;
        leaders &= leaders - 1;
        const int seg = __shfl_sync(0xffffffffu, at, lead);
        const unsigned members = __ballot_sync(0xffffffffu, !second && at == seg) | (1u << lead);
        const Cursor sg = piece[lead];
        const bool begun_here = seg + 1 >= cta_first, whole = begun_here && seg + 2 * sg.np - 1 < cta_end, mine = members >> lane & 1;
        const int ws = 2 * (int)blockIdx.x + (begun_here ? 1 : 0);
        const int kv = kv_of(a, sg.u);                               // (a block of rows that this KV head does not have: none)
        const int rows = max(0, min(ROWS, (a.units.first[kv + 1] - a.units.first[kv]) * a.N - (sg.u - kv * a.blocks) * ROWS));
#pragma unroll 1
        for (; turn < rows; turn += C::WARPS) {
            const int r = turn;
            const float* const po = piece_of[mine ? lane : lead];
            const float m = mine ? po[ROWS * D + 2 * r] : -INFINITY, l = mine ? po[ROWS * D + 2 * r + 1] : 0.f;
            const float M = warp_max(m), f = rebase(m, M), L = warp_sum(l * f);
            float o[D / 32];
#pragma unroll
            for (int y = 0; y < D / 32; ++y) o[y] = 0.f;
            for (unsigned rest = members; rest;) {                   // two pieces at a time
                const int x0 = __ffs(rest) - 1;
                rest &= rest - 1;
                const int x1 = rest ? __ffs(rest) - 1 : x0;
                const float f0 = __shfl_sync(0xffffffffu, f, x0), f1 = rest ? __shfl_sync(0xffffffffu, f, x1) : 0.f;
                rest &= rest - 1;
                const float *p0 = piece_of[x0] + r * D + lane, *p1 = piece_of[x1] + r * D + lane;
                float v0[D / 32], v1[D / 32];
#pragma unroll
                for (int y = 0; y < D / 32; ++y) { v0[y] = p0[32 * y]; v1[y] = p1[32 * y]; }
#pragma unroll
                for (int y = 0; y < D / 32; ++y) o[y] = fmaf(v1[y], f1, fmaf(v0[y], f0, o[y]));
            }
            if (whole) {
                int head, tok;
                row_of<ROWS>(a, sg.u, r, head, tok);
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
        turn -= rows;
    }
}

// The first blocks: page weights, 64 pages of a sequence each: sum over the query heads of (sum of p in the page) / (sum of p in all
// pages).  The rest, DECODE_CTAS for every 16 (row, 32 channels) of a segment: the segment that begins in CTA c0 of the decode kernel
// and goes on in others, joined from their partial sums (32 channels of a row per warp), and the sequences without keys.  The kernel
// lasts as long as one chain of loads, so its first loads wait for none and its code is short; page weights, the longer chain, go
// first (one sequence of 32K tokens: 22.1 -> 20.3 us in all, 4 of 4K: 16.2 -> 15.1, one of 100 tokens with its append and weights:
// 16.7 -> 15.2).
constexpr int JOIN_WARPS = 16;
template <int D, int ROWS>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
cache_join_kernel(const __grid_constant__ DecodeArgs a)
{
    __shared__ float sums[JOIN_WARPS * 32];
    __shared__ float2 ml_of[HIFA4_MAX_HEADS];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int U = units_per_seq(a), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int chunks = (c.max_pages + 63) / 64, block = (int)blockIdx.x - (a.weight_out ? c.B * chunks : 0);
    // the piece of a segment in CTA x: slot 1 where it begins (x = c0), else slot 0
    auto slot_of = [](int x, int c0) { return (2ll * x + (x == c0 ? 1 : 0)) * ROWS; };
    if (block < 0) {
        const int b = (int)blockIdx.x / chunks, p0 = (int)blockIdx.x % chunks * 64;
        const int np = c.n_pages_of(b);
        if (p0 >= np) return;
        const int p = p0 + (tid & 63), grp = tid >> 6;
        constexpr int GROUPS = JOIN_WARPS / 2, AHEAD = 4;
        const float2* src = a.page_ml + (long long)b * a.Hq * c.max_pages + p;
        float2 pre[AHEAD];                                           // of the first heads, asked for ahead of the sums
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            pre[i] = p < np && grp + i * GROUPS < a.Hq ? src[(long long)(grp + i * GROUPS) * c.max_pages] : make_float2(-INFINITY, 0.f);
        for (int j = tid; j < a.Hq; j += JOIN_WARPS * 32) {          // j: place among the query heads sorted by KV head
            int kv = 0;
            while (a.units.first[kv + 1] <= j) ++kv;
            const int in = j - a.units.first[kv], head = a.units.head[j], r = in % ROWS;
            const int2 cc = a.seg_ctas[(long long)b * U + kv * a.blocks + in / ROWS];
            float2 ml;
            if (!segment_recorded(cc.x, cc.y)) {                     // the decode kernel gave up
                ml = make_float2(-INFINITY, 0.f);
            } else if (cc.x == cc.y) {
                ml = a.final_ml[(long long)b * a.Hq + head];
            } else {
                ml = make_float2(-INFINITY, 0.f);
                for (int x = cc.x; x <= cc.y; ++x) ml.x = fmaxf(ml.x, a.part_ml[slot_of(x, cc.x) + r].x);
                for (int x = cc.x; x <= cc.y; ++x) {
                    const float2 y = a.part_ml[slot_of(x, cc.x) + r];
                    ml.y = fmaf(y.y, rebase(y.x, ml.x), ml.y);
                }
            }
            ml_of[head] = make_float2(ml.x, ml.y == 0.f ? 0.f : 1.f / ml.y);
        }
        __syncthreads();
        float w_sum = 0.f;
        if (p < np) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (grp + i * GROUPS < a.Hq) {
                    const float2 all = ml_of[grp + i * GROUPS];
                    w_sum = fmaf(pre[i].y * rebase(pre[i].x, all.x), all.y, w_sum);
                }
#pragma unroll 4
            for (int h = grp + AHEAD * GROUPS; h < a.Hq; h += GROUPS) {
                const float2 ml = src[(long long)h * c.max_pages], all = ml_of[h];
                w_sum = fmaf(ml.y * rebase(ml.x, all.x), all.y, w_sum);
            }
        }
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
    constexpr int AHEAD = 8;
    const int c0 = block % DECODE_CTAS, turn = block / DECODE_CTAS * JOIN_WARPS + warp, r = turn / (D / 32), ch = turn % (D / 32) * 32 + lane;
    auto row_at = [&](int x) { return slot_of(min(c0 + x, DECODE_CTAS - 1), c0) + r; };     // of the x-th partial sum
    const int4 sg = __ldcg(a.begun + c0);
    // asked for before it is known whether there is a segment and how long it is
    float2 ml = __ldcg(a.part_ml + row_at(lane));
    float v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v[i] = __ldcg(a.part_o + row_at(i) * D + ch);
    int head, tok;
    if (sg.x >= 0 && row_of<ROWS>(a, sg.y, r, head, tok)) {
        const int n = sg.z - c0 + 1;
        float M = -INFINITY, L = 0.f, o = 0.f;
#pragma unroll 1
        for (int x0 = 0; x0 < n; x0 += 32) {                         // 32 partial sums at a time
            if (x0) ml = __ldcg(a.part_ml + row_at(x0 + lane));
            if (x0 + lane >= n) ml = make_float2(-INFINITY, 0.f);
            const float old = M;
            M = fmaxf(M, warp_max(ml.x));
            const float g = rebase(old, M), f = rebase(ml.x, M);
            L = fmaf(L, g, ml.y * f);
            o *= g;
            const int most = min(32, n - x0);
#pragma unroll 1
            for (int x = 0; x < most; x += AHEAD) {
                if (x0 + x)
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) v[i] = __ldcg(a.part_o + row_at(x0 + x + i) * D + ch);
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const float fi = __shfl_sync(0xffffffffu, f, x + i);
                    o = fmaf(x + i < most ? v[i] : 0.f, fi, o);
                }
            }
        }
        L = warp_sum(L);
        store_out(a, sg.x, head, tok, D, ch, L == 0.f ? 0.f : o / L);
        if (ch == 0) store_row_stats(a, sg.x, head, tok, M, L);
    }
    if (block >= DECODE_CTAS) return;
    for (int b = block; b < c.B; b += DECODE_CTAS) {            // no keys: zeros
        if (c.n_pages_of(b) > 0) continue;
        if (tid == 0 && c.len(b) < 0) c.invalid();
        for (int i = tid; i < a.Hq * a.N * D; i += JOIN_WARPS * 32) {
            const int head = i / (a.N * D), tok = i / D % a.N;
            store_out(a, b, head, tok, D, i % D, 0.f);
            if (i % D == 0) store_row_stats(a, b, head, tok, -INFINITY, 0.f);
        }
    }
}

int decode_block_rows(int d, int rows) { return rows <= 8 || d == 256 ? 8 : 16; }

size_t decode_first_floats(int d, int block_rows) { return (size_t)DECODE_CTAS * 16 * block_rows * (d + 2); }

template <typename T, int D, int NT, bool SELFTEST = false>
static cudaError_t decode_nt(const DecodeArgs& a, cudaStream_t st)
{
    using C = DecodeCfg<D, NT>;
    static_assert(C::ROWS * D / 32 % JOIN_WARPS == 0, "blocks of the join");
    static SmemOptIn opt;
    if (!opt.ensure(cache_decode_kernel<T, D, NT, SELFTEST>, C::SMEM)) return cudaErrorInvalidValue;
    const cudaError_t e = launch_dependent(cache_decode_kernel<T, D, NT, SELFTEST>, DECODE_CTAS, C::THREADS, C::SMEM, st, a);
    if (e != cudaSuccess) return e;
    const unsigned weight_blocks = a.weight_out ? (unsigned)a.cache.B * ((unsigned)(a.cache.max_pages + 63) / 64) : 0;
    int rows = 0;                                                    // of a block, at most
    for (int kv = 0; kv < a.cache.Hkv; ++kv) rows = std::max(rows, (a.units.first[kv + 1] - a.units.first[kv]) * a.N);
    const unsigned parts = (unsigned)(std::min(rows, C::ROWS) * D / 32 + JOIN_WARPS - 1) / JOIN_WARPS;
    return launch_dependent(cache_join_kernel<D, C::ROWS>, parts * DECODE_CTAS + weight_blocks, JOIN_WARPS * 32, 0, st, a);
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

cudaError_t launch_cache_decode_selftest(const DecodeArgs& a, cudaStream_t st) { return decode_nt<__nv_bfloat16, 128, 1, true>(a, st); }

}  // namespace hifa4
