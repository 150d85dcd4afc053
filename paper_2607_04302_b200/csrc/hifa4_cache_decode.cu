// Attention of a few query rows per KV head over the paged HIF4 cache, split over the caches' lengths and joined.
//
//   S = q~ K^T scale,  m = running max,  p = exp2(S log2e - m + 15),  l = sum p,  O = p V / l
//
// Work: the (sequence, block of query rows of a KV head, page) triples of all sequences, in this order, are dealt out to the
// warps of one CTA per SM in equal contiguous ranges, whatever the sequences' lengths.  A warp takes whole pages on its own:
// it loads them (bulk copies into its own ring), forms S of the page's 64 tokens, its softmax and O, all in registers,
// without any exchange between warps.  The pages of one (sequence, block) that a range holds are a segment; segments that
// warps of one CTA share are joined in shared memory, those that CTAs share by a second, small kernel.
//
// Products run on mma.sync m16n8k16 with the cache as the 16-row operand, tokens (S) or channels (O) its rows, and query rows as the
// 8 columns: an operand of 5 or 6 query rows would leave a 128-row tcgen05 tile nearly empty, and its other operand would have to
// pass through shared memory as 16-bit values, four times the bytes of the codes.  Here codes become MMA operands in
// registers: code * 2^shift (at most 28 in magnitude, exact in FP16 and BF16) by one bit-field insert into the mantissa of
// 2^7 * 2^shift (BF16) or 2^10 * 2^shift (FP16) and one packed add or FMA per two values; the scale of a group multiplies the FP32 sums of the
// group's products, per token for S, per channel for O.  Any order of the contraction index will do as long as both operands
// agree on it, so each lane takes whole 8-code words.
#include "hifa4_cache.cuh"

namespace hifa4 {

using namespace ptx;

template <bool BF>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight codes of a word as four packed pairs (nibble i, nibble i + 4) of code * 2^shift; kk: the two shifts in bits 0-1
// and 16-17.  All steps are exact.
template <bool BF>
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t kk, uint32_t (&r)[4])
{
    if constexpr (BF) {
        const uint32_t one = (kk << 7) + 0x43004300u;                 // 128 * 2^shift, mantissa clear: | nibble = (128 + nibble) * 2^shift
        const uint32_t sub = one + 0x80088008u;                       // -136 * 2^shift
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = ((w >> (4 * i)) & 0x000F000Fu) | one;
            asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(x), "r"(sub));
        }
    } else {
        const uint32_t one = (kk << 10) + 0x64006400u;                // 1024 * 2^shift
        const uint32_t sub = one + 0x80088008u;                       // -1032 * 2^shift
        const uint32_t sub16 = one + 0x70807080u;                     // -72 * 2^shift
        const uint32_t v = w >> 8;
        const uint32_t sixteenth = 0x2C002C00u;
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r[0]) : "r"((w & 0x000F000Fu) | one), "r"(sub));
        r[1] = h2_fma((w & 0x00F000F0u) | one, sixteenth, sub16);     // (1024 + 16 nibble) / 16
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r[2]) : "r"((v & 0x000F000Fu) | one), "r"(sub));
        r[3] = h2_fma((v & 0x00F000F0u) | one, sixteenth, sub16);
    }
}

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
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }

// NT: 8-row column tiles of query rows; H: halves of pages (K, then V) in a warp's ring.
template <int D, int NT> struct DecodeCfg {
    static constexpr int H = D == 256 ? 2 : 4;
    static constexpr int WARPS = D == 256 ? 8 : D == 128 ? (NT == 1 ? 8 : 7) : (NT == 1 ? 12 : 10);
    static constexpr int ROWS = 8 * NT;
    static constexpr int PV_ROW = 36;                                    // words of P per query row: 32 and 4 against bank conflicts
    static constexpr int SLOT = ROWS * (D + 2) * 4;                      // a partial result: O [ROWS][D], then (m, l) [ROWS]
    static constexpr int RING = H * Page<D>::HALF;
    static constexpr int LAST = RING >= SLOT ? 0 : SLOT;                 // the last segment's slot lies over the ring where it fits
    static constexpr int RING_OFF = 0, P_OFF = RING, FIRST_OFF = P_OFF + NT * 8 * PV_ROW * 4;
    static constexpr int LAST_OFF = LAST ? FIRST_OFF + SLOT : RING_OFF;
    static constexpr int PER_WARP = FIRST_OFF + SLOT + LAST;
    static constexpr int BAR_OFF = WARPS * PER_WARP;
    static constexpr int SMEM = BAR_OFF + WARPS * H * 8 + 64;
    static_assert(PER_WARP % 16 == 0 && Page<D>::HALF % 16 == 0 && SMEM <= 227 * 1024, "shared memory");
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
__global__ void __launch_bounds__(DecodeCfg<D, NT>::WARPS * 32, 1)
cache_decode_kernel(const __grid_constant__ DecodeArgs a)
{
    using C = DecodeCfg<D, NT>;
    using P = Page<D>;
    constexpr int NG = P::NG, W = C::WARPS, ROWS = C::ROWS, H = C::H;
    constexpr bool BF = sizeof(T) == 2 && !__is_same(T, __half);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long scratch[W];
    __shared__ Cursor piece[W][2];                     // segments that a warp shares with others: [0] begun before it, [1] in it
    __shared__ long long piece_at[W][2];               // index of the segment's first page in the list of work, -1: no such piece
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const uint32_t base = smem_u32(smem) + warp * C::PER_WARP;
    const uint32_t ring = base + C::RING_OFF, pbuf = base + C::P_OFF;
    const uint32_t bars = smem_u32(smem) + C::BAR_OFF + warp * H * 8;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < H; ++i) mbar_init(bars + 8 * i, 1);
        fence_barrier_init();
    }
    if (lane < 2) piece_at[warp][lane] = -1;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int U = units_per_seq(a);
    const long long total = pages_before(c, c.B, scratch) * U;
    const int ctas = active_ctas(total);
    if ((int)blockIdx.x >= ctas) return;
    const long long nw = (long long)ctas * W;
    const long long cta0 = total * blockIdx.x / ctas, cta1 = total * (blockIdx.x + 1) / ctas;
    const long long w0 = total * ((long long)blockIdx.x * W + warp) / nw, w1 = total * ((long long)blockIdx.x * W + warp + 1) / nw;
    int remaining = (int)(w1 - w0);

    // where the range begins
    Cursor cur{0, 0, 0, 0};
    long long seg_at = w0;                             // index of the present segment's first page
    if (remaining > 0) {
        long long before = 0;
        for (int b0 = 0; b0 < c.B; b0 += 32) {
            const int np = b0 + lane < c.B ? c.n_pages_of(b0 + lane) : 0;
            int pre = np;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, pre, o);
                if (lane >= o) pre += x;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, (before + pre) * U > w0);
            if (hit) {
                const int l = __ffs(hit) - 1;
                cur.b = b0 + l;
                cur.np = __shfl_sync(0xffffffffu, np, l);
                before += __shfl_sync(0xffffffffu, pre - np, l);
                break;
            }
            before += __shfl_sync(0xffffffffu, pre, 31);
        }
        const long long in = w0 - before * U;
        cur.u = (int)(in / cur.np);
        cur.p = (int)(in % cur.np);
        seg_at = w0 - cur.p;
    }

    // loader: runs ahead of the computation by up to H half pages; 32 page numbers at a time
    Cursor ld = cur;
    int ids = 0, ids_at = -1, ids_b = -1, loaded = 0;  // loaded: half pages asked for
    uint32_t there_bits = 0;                           // bit i % 32: page i of the range exists
    const int halves = 2 * remaining;
    auto load_next = [&]() {
        if (loaded >= halves) return;
        if (!(loaded & 1) && (ids_b != ld.b || (ld.p & ~31) != ids_at)) {
            ids_b = ld.b;
            ids_at = ld.p & ~31;
            ids = ids_at + lane < ld.np ? c.page(ld.b, ids_at + lane) : -1;
        }
        const int page = __shfl_sync(0xffffffffu, ids, ld.p & 31);
        const int st = loaded % H;
        if (!(loaded & 1)) there_bits = (there_bits & ~(1u << (loaded / 2 % 32))) | (page >= 0 ? 1u << (loaded / 2 % 32) : 0u);
        if (lane == 0) {
            if (page >= 0) {
                mbar_expect_tx(bars + 8 * st, P::HALF);
                bulk_load(ring + st * P::HALF,
                          c.pages + ((long long)page * c.Hkv + ld.u / a.blocks) * P::BYTES + (loaded & 1) * P::HALF, P::HALF, bars + 8 * st);
            } else {
                mbar_arrive(bars + 8 * st);            // nothing to load: the tokens are left out
            }
        }
        if (loaded & 1) {
            if (++ld.p == ld.np) {
                ld.p = 0;
                if (++ld.u == U) {
                    ld.u = 0;
                    do { ++ld.b; } while (ld.b < c.B && (ld.np = c.n_pages_of(ld.b)) == 0);
                }
            }
        }
        ++loaded;
    };
#pragma unroll 1
    for (int i = 0; i < H; ++i) load_next();

    int done = 0;                                      // half pages consumed
    bool ok = true;
#pragma unroll 1
    while (remaining > 0 && ok) {
        // ---- a segment: query operands
        const int kv = cur.u / a.blocks, len = c.len(cur.b);
        uint32_t qf[NT][NG][4][2];
        int limit[NT][2];                              // keys that the rows of columns 2t, 2t + 1 see
        int full = len;                                // keys that every row sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int head = 0, tok = 0;
            const bool have = row_of<ROWS>(a, cur.u, nt * 8 + g, head, tok);
            const uint16_t* qp = (const uint16_t*)a.q + cur.b * a.qs.b + head * a.qs.h + tok * a.qs.t;
#pragma unroll
            for (int G = 0; G < NG; ++G) {
                uint32_t x[8] = {0, 0, 0, 0, 0, 0, 0, 0};           // elements 16t..16t+15 of the group
                if (have) {
                    const uint4 lo = __ldg(reinterpret_cast<const uint4*>(qp + 64 * G + 16 * t));
                    const uint4 hi = __ldg(reinterpret_cast<const uint4*>(qp + 64 * G + 16 * t) + 1);
                    x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w;
                    x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
                    if (a.s) {                                      // FP32 product, rounded once to the activation dtype
                        const float4* sp = reinterpret_cast<const float4*>(a.s + kv * D + 64 * G + 16 * t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 f = __ldg(sp + i);
                            float e0, e1;
                            Pair16<T>::unpack(x[2 * i], e0, e1);
                            x[2 * i] = Pair16<T>::round_pack(e0 * f.x, e1 * f.y);
                            Pair16<T>::unpack(x[2 * i + 1], e0, e1);
                            x[2 * i + 1] = Pair16<T>::round_pack(e0 * f.z, e1 * f.w);
                        }
                    }
                }
                // pairs (i, i + 4) of each unit
                qf[nt][G][0][0] = __byte_perm(x[0], x[2], 0x5410); qf[nt][G][1][0] = __byte_perm(x[0], x[2], 0x7632);
                qf[nt][G][2][0] = __byte_perm(x[1], x[3], 0x5410); qf[nt][G][3][0] = __byte_perm(x[1], x[3], 0x7632);
                qf[nt][G][0][1] = __byte_perm(x[4], x[6], 0x5410); qf[nt][G][1][1] = __byte_perm(x[4], x[6], 0x7632);
                qf[nt][G][2][1] = __byte_perm(x[5], x[7], 0x5410); qf[nt][G][3][1] = __byte_perm(x[5], x[7], 0x7632);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                limit[nt][e] = len;
                if (a.causal && row_of<ROWS>(a, cur.u, nt * 8 + 2 * t + e, head, tok)) {
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
            int st = done % H;
            uint32_t kb = ring + st * P::HALF;
            if (!__all_sync(0xffffffffu, mbar_wait(bars + 8 * st, (done / H) & 1))) { ok = false; break; }
            const bool there = there_bits >> (done / 2 % 32) & 1u;
            float s[4][NT][4];
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
                        sc[r][G] = quarter_scale(lds8(kb + P::K_SCALES + row * NG + G));
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
                        const uint32_t y = shw[r][G] >> (4 * t);
                        unpack8<BF>(w[r][G][0], y & 0x00030003u, A[r][0]);
                        unpack8<BF>(w[r][G][1], (y >> 2) & 0x00030003u, A[r][1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma16816<BF>(acc, A[0][0][x], A[1][0][x], A[0][1][x], A[1][1][x], qf[nt][G][x][0], qf[nt][G][x][1]);
                        s[i][nt][0] = fmaf(acc[0], sc[0][G], s[i][nt][0]);
                        s[i][nt][1] = fmaf(acc[1], sc[0][G], s[i][nt][1]);
                        s[i][nt][2] = fmaf(acc[2], sc[1][G], s[i][nt][2]);
                        s[i][nt][3] = fmaf(acc[3], sc[1][G], s[i][nt][3]);
                    }
                }
            }
            __syncwarp();
            ++done;
            load_next();
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
                    const float mn = fmaxf(m[nt][e], fmaf(mx, a.scale_log2, -15.f));
                    const float ref = mn == -INFINITY ? 0.f : mn;
                    f[nt][e] = ex2_approx(m[nt][e] - ref);
                    moved |= mn != m[nt][e];
                    m[nt][e] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = ex2_approx(fmaf(s[i][nt][e], a.scale_log2, -ref));
                        const float p1 = ex2_approx(fmaf(s[i][nt][e + 2], a.scale_log2, -ref));
                        sum += p0 + p1;
                        pw[nt][e][i] = Pair16<__half>::round_pack(p0, p1);
                    }
                    l[nt][e] = fmaf(l[nt][e], f[nt][e], sum);
                    if (a.page_ml) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                        int head, tok;
                        if (g == 0 && row_of<ROWS>(a, cur.u, nt * 8 + 2 * t + e, head, tok))
                            a.page_ml[((long long)cur.b * a.Hq + head) * c.max_pages + p] = make_float2(mn, sum);
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
            st = done % H;
            const uint32_t vb = ring + st * P::HALF;
            if (!__all_sync(0xffffffffu, mbar_wait(bars + 8 * st, (done / H) & 1))) { ok = false; break; }
            if (there) {
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    uint32_t A[2][2][4];
                    float sc[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int ch = 16 * j + 8 * r + g;
                        const uint2 w = lds64(vb + P::K_CODES + ch * 32 + t * 8);
                        const uint32_t y = lds32(vb + P::K_SHIFTS + 4 * ch) >> (4 * t);
                        sc[r] = quarter_scale(lds8(vb + P::K_SCALES + ch));
                        unpack8<false>(w.x, y & 0x00030003u, A[r][0]);
                        unpack8<false>(w.y, (y >> 2) & 0x00030003u, A[r][1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma16816<false>(acc, A[0][0][x], A[1][0][x], A[0][1][x], A[1][1][x], pf[nt][x], pf[nt][4 + x]);
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
            ++done;
            load_next();
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
            float* po = reinterpret_cast<float*>(smem + warp * C::PER_WARP + (slot ? C::LAST_OFF : C::FIRST_OFF));
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
                piece[warp][slot] = cur;
                piece_at[warp][slot] = seg_at;
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
        if (lane == 0 && c.d_status) *c.d_status = HIFA4_ERR_TIMEOUT;
        let_copies_land();
    }
    // ---- segments that warps share
    __syncthreads();
#pragma unroll 1
    for (int w = 0; w < W; ++w)
#pragma unroll 1
        for (int slot = 0; slot < 2; ++slot) {
            const long long at = piece_at[w][slot];
            if (at < 0) continue;
            if (slot == 0 && at >= cta0) continue;                   // joined where the segment begins
            if (slot == 0) {                                         // begun before this CTA: its first piece here
                bool earlier = false;
                for (int x = 0; x < w; ++x) earlier |= piece_at[x][0] == at;
                if (earlier) continue;
            }
            const Cursor sg = piece[w][slot];
            int end = w + 1;                                         // warps [w, end) hold it
            for (int x = w + 1; x < W; ++x)
                if (piece_at[x][0] == at) end = x + 1;
            const bool whole = at >= cta0 && at + sg.np <= cta1;
            const int ws = 2 * (int)blockIdx.x + (at < cta0 ? 0 : 1);
            auto slot_of = [&](int x) {
                return reinterpret_cast<const float*>(smem + x * C::PER_WARP + (x == w && slot ? C::LAST_OFF : C::FIRST_OFF));
            };
            for (int i = tid; i < ROWS * D; i += W * 32) {
                const int r = i / D, ch = i % D;
                int head, tok;
                if (!row_of<ROWS>(a, sg.u, r, head, tok)) break;     // rows only grow
                float M = -INFINITY;
                for (int x = w; x < end; ++x)
                    if (x == w || piece_at[x][0] == at) M = fmaxf(M, slot_of(x)[ROWS * D + 2 * r]);
                float L = 0.f, O = 0.f;
                for (int x = w; x < end; ++x)
                    if (x == w || piece_at[x][0] == at) {
                        const float* po = slot_of(x);
                        const float fx = rebase(po[ROWS * D + 2 * r], M);
                        L = fmaf(po[ROWS * D + 2 * r + 1], fx, L);
                        O = fmaf(po[i], fx, O);
                    }
                if (whole) {
                    store_out(a, sg.b, head, tok, D, ch, L == 0.f ? 0.f : O / L);
                    if (ch == 0) store_row_stats(a, sg.b, head, tok, M, L);
                } else {
                    a.part_o[(long long)ws * ROWS * D + i] = O;
                    if (ch == 0) a.part_ml[(long long)ws * ROWS + r] = make_float2(M, L);
                }
            }
        }
}

// Segments that CTAs share, and sequences without keys.  One block of D threads per (sequence, unit).
template <int D, int ROWS>
__global__ void __launch_bounds__(D)
cache_join_kernel(const __grid_constant__ DecodeArgs a)
{
    __shared__ long long scratch[D / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int U = units_per_seq(a), b = blockIdx.x / U, u = blockIdx.x % U, ch = threadIdx.x;
    const int np = c.n_pages_of(b);
    if (u == 0 && ch == 0 && c.len(b) < 0) c.invalid();
    long long at = 0, c0 = 0, c1 = 0;
    if (np > 0) {
        const long long total = pages_before(c, c.B, scratch) * U;
        at = pages_before(c, b, scratch) * U + (long long)u * np;
        const int ctas = active_ctas(total);
        c0 = ((at + 1) * ctas - 1) / total;                          // CTAs of the first and the last page
        c1 = ((at + np) * ctas - 1) / total;
        if (c0 == c1) return;
    }
    for (int r = 0; r < ROWS; ++r) {
        int head, tok;
        if (!row_of<ROWS>(a, u, r, head, tok)) return;
        float M = -INFINITY, L = 0.f, O = 0.f;
        if (np > 0) {
            for (long long x = c0; x <= c1; ++x) M = fmaxf(M, a.part_ml[(2 * x + (x == c0 ? 1 : 0)) * ROWS + r].x);
            for (long long x = c0; x <= c1; ++x) {
                const long long ws = 2 * x + (x == c0 ? 1 : 0);
                const float2 ml = a.part_ml[ws * ROWS + r];
                const float fx = rebase(ml.x, M);
                L = fmaf(ml.y, fx, L);
                O = fmaf(a.part_o[(ws * ROWS + r) * D + ch], fx, O);
            }
        }
        store_out(a, b, head, tok, D, ch, L == 0.f ? 0.f : O / L);
        if (ch == 0) store_row_stats(a, b, head, tok, M, L);
    }
}

// Weights of the pages: sum over the query heads of (sum of p in the page) / (sum of p in all pages).  A thread per page.
__global__ void __launch_bounds__(128)
cache_weight_kernel(const __grid_constant__ DecodeArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const CacheView& c = a.cache;
    const int b = blockIdx.y, p = blockIdx.x * 128 + threadIdx.x;
    if (p >= c.n_pages_of(b)) return;
    float w = 0.f;
    for (int h = 0; h < a.Hq; ++h) {
        const float2 all = a.final_ml[(long long)b * a.Hq + h];
        const float2 ml = a.page_ml[((long long)b * a.Hq + h) * c.max_pages + p];
        if (all.y != 0.f) w += ml.y * rebase(ml.x, all.x) / all.y;
    }
    const long long i = (long long)b * c.max_pages + p;
    a.weight_out[i] = (a.weight ? a.weight[i] : 0.f) + w;
}

int decode_block_rows(int d, int rows) { return rows <= 8 || d == 256 ? 8 : 16; }

template <typename T, int D, int NT>
static cudaError_t decode_nt(const DecodeArgs& a, cudaStream_t st)
{
    using C = DecodeCfg<D, NT>;
    static SmemOptIn opt;
    if (!opt.ensure(cache_decode_kernel<T, D, NT>, C::SMEM)) return cudaErrorInvalidValue;
    cudaError_t e = launch_dependent(cache_decode_kernel<T, D, NT>, DECODE_CTAS, C::WARPS * 32, C::SMEM, st, a);
    if (e != cudaSuccess) return e;
    e = launch_dependent(cache_join_kernel<D, C::ROWS>, (unsigned)(a.cache.B * a.cache.Hkv * a.blocks), D, 0, st, a);
    if (e != cudaSuccess || !a.weight_out) return e;
    return launch_dependent(cache_weight_kernel, dim3((unsigned)(a.cache.max_pages + 127) / 128, (unsigned)a.cache.B), 128, 0, st, a);
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
