// Attention of many query rows over the paged HIF4 cache on tcgen05 (cross attention, chunks of a prompt).
//
//   S = Q~ K^T scale,  m = running reference,  P = exp2(S log2e - m),  O += P V,  l += sum P,  out = O / l
//
// One CTA per 256 (QT = 2) or 128 query rows of one KV head and sequence, or per a share of the sequence's pages for the blocks of
// a last wave that would not fill the chip (joined by a second kernel).  Rows are (query head, token) pairs in the order of the
// heads, so that short queries of several heads fill a tile.  Key tiles are pages.  With 128 rows or fewer to a CTA of two tiles,
// both take the same rows, one the even and one the odd pages, and are joined in shared memory: what bounds such a CTA is the
// chain of a tile from page to page.
//
// Both products take the exact BF16 values of the cache, which dequantization warps write to shared memory from the pages' codes:
// an image of the cache in global memory would be 3.5 times its size, and only 15 instructions per 8 values are needed, a quarter
// of what the softmax of 256 rows executes meanwhile.  Q~ is the first operand of S from tensor memory (an M = 128, N = 64 MMA takes 32 clk
// with the first operand there, 48 with it in shared memory), P that of O.  P is rounded to BF16; for FP16 activations Q~ and P are
// split into two BF16 terms each (16 bits), and both products take two MMAs.
// The reference of a row moves only when its maximum exceeds it by more than 2^8: P stays below 2^8, FP32 sums hold, and O is
// rarely rescaled.
//
// Warps: 0-3 (and 4-7) softmax of a tile, one thread per row; the next four dequantize; then an issuer of MMAs per tile, which waits
// for its tile alone and suspended in hardware (one that polls for both tiles takes issue slots from the softmax warps of its
// scheduler, one that takes them in turn makes each wait for the other), and the loader.
// S is released as soon as it is in registers, so that the next S is formed under the softmax; P has columns of its own.  Order
// among MMAs of different shapes is not relied on: every reuse of tensor memory waits for a commit.
#include <type_traits>

#include "hifa4_cache.cuh"
#include "hifa4_ptx.cuh"

namespace hifa4 {

template <int D, bool SPLIT> struct TileCfg {
    static constexpr int NG = D / 64, TERMS = SPLIT ? 2 : 1;
    static constexpr int QT = D == 64 || (D == 128 && !SPLIT) ? 2 : 1;
    static constexpr int P_COLS = 32 * TERMS;
    // tensor memory: O, S and P of the tiles, then the terms of Q~ that fit; the others are in shared memory
    static constexpr int S_COL = QT * D, P_COL = S_COL + QT * 64, Q_COL = P_COL + QT * P_COLS;
    static constexpr int Q_FIT = (512 - Q_COL) / (D / 2);
    static constexpr int Q_SMEM = QT * TERMS > Q_FIT ? QT * TERMS - Q_FIT : 0;      // (tile, term) pairs, the last ones
    static constexpr int SMW = 4 * QT, W_DQ = SMW, W_MMA = SMW + 4, W_LD = W_MMA + QT, THREADS = (W_LD + 1) * 32;
    static constexpr int KS = D == 256 ? 2 : 3;                          // stages of K and V tiles
    static constexpr int RS = D == 256 ? (SPLIT ? 1 : 2) : 3;            // of raw pages
    static constexpr int K_STAGE = 64 * D * 2, V_STAGE = D * 128, Q_TERM = 128 * D * 2;
    static constexpr int V_OFF = KS * K_STAGE, Q_OFF = V_OFF + KS * V_STAGE, RAW_OFF = Q_OFF + Q_SMEM * Q_TERM;
    static constexpr int MISC_OFF = RAW_OFF + RS * Page<D>::BYTES;
    static constexpr int SMEM = MISC_OFF + 512 + 1024;
    static_assert(SMEM <= 226 * 1024 && Page<D>::BYTES % 16 == 0, "shared memory");
};

namespace tilek {
// RF / RE raw page landed / read; KF / KE, VF / VE tile written / read by the MMAs; QF Q~ stored; per tile: SF S complete, SR S in
// registers, PF P stored, OD O complete.
enum { RF = 0, RE = 3, KF = 6, KE = 9, VF = 12, VE = 15, QF = 18, SF = 20, SR = 22, PF = 24, OD = 26, N_BARS = 28 };
constexpr uint32_t POLLS = 1u << 18;
constexpr int POLY = 1;
}  // namespace tilek

__device__ __forceinline__ bool tile_wait(uint32_t bar, uint32_t parity, volatile int* abort, uint32_t polls = tilek::POLLS)
{
#pragma unroll 1
    for (uint32_t i = 0; i < polls; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 63u && *abort) return false;
    }
    return false;
}

// Two exponentials to base 2 on the multiply-add pipe, for -126 <= x (less counts as -126) and x < 127: x = n + f with n the nearest
// integer (by adding 1.5 * 2^23, whose low bits then hold n), 2^f by the polynomial of degree 5 that has the least largest relative
// error on [-1/2, 1/2] (fitted by reweighted least squares; 2.15e-7 with FP32 coefficients and Horner steps), n added to the exponent.
__device__ __forceinline__ void exp2_pair(float& x0, float& x1)
{
    const uint64_t magic = pack2(12582912.f, 12582912.f), unmagic = pack2(-12582912.f, -12582912.f), minus = pack2(-1.f, -1.f);
    const uint64_t x = pack2(fmaxf(x0, -126.f), fmaxf(x1, -126.f)), t = add2(x, magic), f = fma2(add2(t, unmagic), minus, x);
    uint64_t p = pack2(0.0013276472454890609f, 0.0013276472454890609f);
    p = fma2(p, f, pack2(0.009675540961325169f, 0.009675540961325169f));
    p = fma2(p, f, pack2(0.05550713092088699f, 0.05550713092088699f));
    p = fma2(p, f, pack2(0.24022120237350464f, 0.24022120237350464f));
    p = fma2(p, f, pack2(0.6931469440460205f, 0.6931469440460205f));
    p = fma2(p, f, pack2(1.0000001192092896f, 1.0000001192092896f));
    float p0, p1, t0, t1;
    unpack2(p, p0, p1);
    unpack2(t, t0, t1);
    uint32_t r0, r1;
    asm("mad.lo.u32 %0, %1, 0x800000, %2;" : "=r"(r0) : "r"(__float_as_uint(t0)), "r"(__float_as_uint(p0)));
    asm("mad.lo.u32 %0, %1, 0x800000, %2;" : "=r"(r1) : "r"(__float_as_uint(t1)), "r"(__float_as_uint(p1)));
    x0 = __uint_as_float(r0);
    x1 = __uint_as_float(r1);
}

__device__ __forceinline__ void tile_store(const TileArgs& a, long long i, float x, float y)
{
    if (a.out_dtype == HIFA4_BF16) ((uint32_t*)a.out)[i / 2] = Pair16<__nv_bfloat16>::round_pack(x, y);
    else if (a.out_dtype == HIFA4_F16) ((uint32_t*)a.out)[i / 2] = Pair16<__half>::round_pack(x, y);
    else ((float2*)a.out)[i / 2] = make_float2(x, y);
}
template <typename O> __device__ __forceinline__ void store32_16(void* out, long long i, const uint32_t (&o)[32])
{
    uint4* dst = reinterpret_cast<uint4*>((uint16_t*)out + i);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        uint32_t v[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) v[y] = Pair16<O>::round_pack(__uint_as_float(o[8 * x + 2 * y]), __uint_as_float(o[8 * x + 2 * y + 1]));
        dst[x] = make_uint4(v[0], v[1], v[2], v[3]);
    }
}
__device__ __forceinline__ void tile_store32(const TileArgs& a, long long i, const uint32_t (&o)[32])   // 32 values of a row
{
    if (a.out_dtype == HIFA4_BF16) store32_16<__nv_bfloat16>(a.out, i, o);
    else if (a.out_dtype == HIFA4_F16) store32_16<__half>(a.out, i, o);
    else {
        uint4* dst = reinterpret_cast<uint4*>((float*)a.out + i);
#pragma unroll
        for (int x = 0; x < 8; ++x) dst[x] = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
    }
}

// SELFTEST (hifa4_selftest_cache_wait_timeout): the first CTA's loader leaves its third page out, and the warps that wait for it give
// up after 2^6 polls.
template <typename T, int D, bool SELFTEST>
__global__ void __launch_bounds__(TileCfg<D, __is_same(T, __half)>::THREADS, 1)
cache_attention_kernel(const __grid_constant__ TileArgs a)
{
    constexpr bool SPLIT = __is_same(T, __half);
    using C = TileCfg<D, SPLIT>;
    using P = Page<D>;
    using namespace tilek;
    constexpr int NG = C::NG;
    extern __shared__ uint8_t smem_raw[];
    __shared__ volatile int abort_flag;
    __shared__ volatile int there[16];                               // whether page j exists: entry j % 16
    __shared__ uint32_t tmem_slot;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bars = smem + C::MISC_OFF;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < 3; ++i) {
            mbar_init(bar(RF + i), 1); mbar_init(bar(RE + i), 4);
            mbar_init(bar(KF + i), 4); mbar_init(bar(KE + i), C::QT);
            mbar_init(bar(VF + i), 4); mbar_init(bar(VE + i), C::QT);
        }
        mbar_init(bar(QF), C::SMW);
        for (int i = 0; i < 2; ++i) { mbar_init(bar(SF + i), 1); mbar_init(bar(SR + i), 4); mbar_init(bar(PF + i), 4); mbar_init(bar(OD + i), 1); }
        fence_barrier_init();
        abort_flag = 0;
    }
    // Tensor memory is taken when the kernel before is over, and the next one may start when every CTA has its own: of two kernels
    // on an SM none waits for columns that the other holds while it waits for the whole grid.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == C::W_MMA) { tmem_alloc(smem_u32(&tmem_slot), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    const CacheView& c = a.cache;
    int w = blockIdx.x, sp = 0, splits = 1;
    if (w >= a.full) {                                               // a block of the last wave: its pages are shared out
        splits = a.splits;
        sp = (w - a.full) % splits;
        w = a.full + (w - a.full) / splits;
    }
    const int slot = w - a.full;                                     // of its partial results
    const int item = a.items - 1 - w % a.items; w /= a.items;        // causal: the longest rows first
    const int kv = w % c.Hkv, b = w / c.Hkv;
    const int len = max(c.len(b), 0);
    const int rows = (a.units.first[kv + 1] - a.units.first[kv]) * a.N, row0 = item * 128 * C::QT;
    const int tiles = row0 >= rows ? 0 : C::QT == 2 && row0 + 128 < rows ? 2 : 1;
    int seen = len;                                                  // keys that some row sees
    if (a.causal && tiles) {
        const int last = min(rows, row0 + 128 * C::QT) - 1;
        const int tok = last / a.N > row0 / a.N ? a.N - 1 : last % a.N;      // the block's last token of any head
        seen = min(len, max(0, len - a.N + 1 + tok));
    }
    const int np = (seen + 63) >> 6, j0 = (int)((long long)np * sp / splits), j1 = (int)((long long)np * (sp + 1) / splits);
    const int n = tiles ? j1 - j0 : 0;
    const bool alt = C::QT == 2 && tiles == 1;                       // both tiles take these rows, tile h the pages h, h + 2, ..
    if (tid == 0 && item == 0 && kv == 0 && sp == 0 && c.len(b) < 0) c.invalid();

    auto fail = [&]() {
        abort_flag = 1;
        c.timed_out();
    };
    bool ok = true;

    // softmax warps: the thread's row
    const int h_sm = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + (alt ? 0 : 128 * h_sm) + r;
    const bool have = warp < C::SMW && row < rows;
    const int head = have ? a.units.head[a.units.first[kv] + row / a.N] : 0, tok = have ? row % a.N : 0;
    float m = -INFINITY, l = 0.f;
    const int n_tile = alt ? (n + 1 - h_sm) >> 1 : h_sm < tiles ? n : 0;          // pages of the warp's tile

    if (warp < C::SMW) {
        // ------------------------------------------------------------------ softmax: a row per thread
        const int h = h_sm;
        const uint32_t t_w = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_o = t_w + h * D, t_s = t_w + C::S_COL + 64 * h,
                       t_p = t_w + C::P_COL + C::P_COLS * h;
        const int limit = !have ? 0 : a.causal ? len - a.N + 1 + tok : len;
        if (n_tile > 0) {
            const uint16_t* qp = (const uint16_t*)a.q + b * a.qs.b + head * a.qs.h + tok * a.qs.t;
#pragma unroll 1
            for (int G = 0; G < NG; ++G) {
                uint32_t hi[32], lo[32];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (have) v = __ldg(reinterpret_cast<const uint4*>(qp + 64 * G) + u);
                    uint32_t x[4] = {v.x, v.y, v.z, v.w}, y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float e0, e1;
                        Pair16<T>::unpack(x[i], e0, e1);
                        if (a.s) {                                   // FP32 product, rounded once to the activation dtype
                            const float2 f = __ldg(reinterpret_cast<const float2*>(a.s + kv * D + 64 * G + 8 * u) + i);
                            Pair16<T>::unpack(Pair16<T>::round_pack(e0 * f.x, e1 * f.y), e0, e1);
                        }
                        x[i] = Pair16<__nv_bfloat16>::round_pack(e0, e1);
                        if (SPLIT) {
                            float h0, h1;
                            Pair16<__nv_bfloat16>::unpack(x[i], h0, h1);
                            y[i] = Pair16<__nv_bfloat16>::round_pack(e0 - h0, e1 - h1);
                        }
                    }
                    // the order of the dequantized keys: pairs (i, i + 4)
                    hi[4 * u] = __byte_perm(x[0], x[2], 0x5410); hi[4 * u + 1] = __byte_perm(x[0], x[2], 0x7632);
                    hi[4 * u + 2] = __byte_perm(x[1], x[3], 0x5410); hi[4 * u + 3] = __byte_perm(x[1], x[3], 0x7632);
                    if (SPLIT) {
                        lo[4 * u] = __byte_perm(y[0], y[2], 0x5410); lo[4 * u + 1] = __byte_perm(y[0], y[2], 0x7632);
                        lo[4 * u + 2] = __byte_perm(y[1], y[3], 0x5410); lo[4 * u + 3] = __byte_perm(y[1], y[3], 0x7632);
                    }
                }
                auto put = [&](int term, const uint32_t (&v)[32]) {
                    const int i = h * C::TERMS + term;
                    if (i < C::Q_FIT) {
                        tmem_st32(t_w + C::Q_COL + i * (D / 2) + 32 * G, v);
                        return;
                    }
                    const uint32_t at = smem + C::Q_OFF + (i - C::Q_FIT) * C::Q_TERM + G * 16384 + r * 128;
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + ((uint32_t)(u ^ (r & 7)) << 4)), "r"(v[4 * u]),
                                     "r"(v[4 * u + 1]), "r"(v[4 * u + 2]), "r"(v[4 * u + 3]) : "memory");
                };
                put(0, hi);
                if (SPLIT) put(1, lo);
            }
            tmem_wait_st();
            fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(QF));
        if (n_tile > 0) {
            const int full = a.causal ? __reduce_min_sync(0xffffffffu, have ? limit : len) : len;      // keys that every row of the warp sees
#pragma unroll 1
            for (int j = 0; j < n_tile; ++j) {
                if (!__all_sync(0xffffffffu, tile_wait(bar(SF + h), (uint32_t)j & 1u, &abort_flag))) { fail(); ok = false; break; }
                tc_fence_after();
                uint32_t sr[2][32];
                tmem_ld32(t_s, sr[0]);
                tmem_ld32(t_s + 32, sr[1]);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(SR + h));
                const int pg = alt ? 2 * j + h : j, k0 = 64 * (j0 + pg);
                const bool page = there[pg & 15];
                const bool masked = k0 + 64 > full || !page;
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (!page || k0 + i >= limit) sr[i >> 5][i & 31] = 0xFF800000u;
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 64; i += 8)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        mx[y] = max3(mx[y], __uint_as_float(sr[i >> 5][(i & 31) + 2 * y]), __uint_as_float(sr[i >> 5][(i & 31) + 2 * y + 1]));
                const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * a.scale_log2;
                const bool plain = !masked && __all_sync(0xffffffffu, fabsf(top) < INFINITY);
                const bool move = top > m + 8.f;
                float rescale = 1.f;
                const bool moved = __any_sync(0xffffffffu, move);
                if (moved) {
                    const float f = !move ? 1.f : m == -INFINITY ? 0.f : ex2_approx(m - top);
                    if (move) m = top;
                    l *= f;
                    rescale = f;
                }
                const float ref = m == -INFINITY ? 0.f : m;
                const uint64_t c2 = pack2(a.scale_log2, a.scale_log2), r2 = pack2(-ref, -ref);
                uint64_t sum[2] = {0, 0};
                float* const x = reinterpret_cast<float*>(&sr[0][0]);
                // The special-function unit gives 16 exponentials per clk and SM, 1024 clk for the page's: POLY of four pairs go to the
                // multiply-add pipe, unless a score is masked or not finite (exp2_pair has no zero).
                auto exponentials = [&](auto poly) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float p0, p1;
                        unpack2(fma2(pack2(x[2 * i], x[2 * i + 1]), c2, r2), p0, p1);
                        if (decltype(poly)::value && i % 4 >= 4 - POLY) {
                            exp2_pair(p0, p1);
                        } else {
                            p0 = ex2_approx(p0);
                            p1 = ex2_approx(p1);
                        }
                        sum[i & 1] = add2(sum[i & 1], pack2(p0, p1));
                        x[2 * i] = p0;
                        x[2 * i + 1] = p1;
                    }
                };
                if (plain) exponentials(std::true_type{});
                else exponentials(std::false_type{});
                // word 8 i + e of P: tokens 16 i + e and 16 i + 8 + e, the order of the dequantized values
                uint32_t ps[32], pl[32];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float p0 = x[16 * i + e], p1 = x[16 * i + 8 + e];
                        const uint32_t hi = Pair16<__nv_bfloat16>::round_pack(p0, p1);
                        ps[8 * i + e] = hi;
                        if (SPLIT) {
                            float h0, h1;
                            Pair16<__nv_bfloat16>::unpack(hi, h0, h1);
                            pl[8 * i + e] = Pair16<__nv_bfloat16>::round_pack(p0 - h0, p1 - h1);
                        }
                    }
                float s0, s1;
                unpack2(add2(sum[0], sum[1]), s0, s1);
                l += s0 + s1;
                if (j > 0) {                                         // P(j - 1) is read and O complete
                    if (!__all_sync(0xffffffffu, tile_wait(bar(OD + h), (uint32_t)(j - 1) & 1u, &abort_flag))) { fail(); ok = false; break; }
                    tc_fence_after();
                }
                tmem_st32(t_p, ps);
                if (SPLIT) tmem_st32(t_p + 32, pl);
                if (moved && j > 0) {
#pragma unroll 1
                    for (int y = 0; y < D; y += 32) {
                        uint32_t o[32];
                        tmem_ld32(t_o + y, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * rescale);
                        tmem_st32(t_o + y, o);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(PF + h));
            }
        }
    } else if (warp < C::W_MMA) {
        // ------------------------------------------------------------------ codes -> BF16 tiles
        const int dw = warp - C::W_DQ, sub = lane >> 2, p = lane & 3;
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            const int rs = j % C::RS, ks = j % C::KS;
            const uint32_t raw = smem + C::RAW_OFF + rs * P::BYTES, k_t = smem + ks * C::K_STAGE, v_t = smem + C::V_OFF + ks * C::V_STAGE;
            const uint32_t free_ph = (uint32_t)(j / C::KS + 1) & 1u;           // the first round passes
            if (!__all_sync(0xffffffffu, tile_wait(bar(RF + rs), (uint32_t)(j / C::RS) & 1u, &abort_flag,
                                                   SELFTEST && blockIdx.x == 0 && j == 2 ? 1u << 6 : POLLS) &&
                                             tile_wait(bar(KE + ks), free_ph, &abort_flag))) { fail(); ok = false; break; }
            // K: a lane takes the units 2 p, 2 p + 1 of every group of a row
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const int row = 32 * it + 8 * dw + sub;
#pragma unroll
                for (int G = 0; G < NG; ++G) {
                    uint32_t w0, w1, sh, sc, o[4];
                    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w0), "=r"(w1) : "r"(raw + P::K_CODES + row * (D / 2) + p * 8 * NG + 8 * G));
                    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sh) : "r"(raw + P::K_SHIFTS + 4 * (row * NG + G)));
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(sc) : "r"(raw + P::K_SCALES + row * NG + G));
                    const uint32_t y = shifts_of_unit(sh, 2 * p), s2 = scale_pair(sc), dst = k_t + G * 8192 + row * 128;
                    hif4_word_values(w0, y, s2, o);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + ((uint32_t)((2 * p) ^ (row & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                                 "r"(o[2]), "r"(o[3]) : "memory");
                    hif4_word_values(w1, y >> 2, s2, o);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + ((uint32_t)((2 * p + 1) ^ (row & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                                 "r"(o[2]), "r"(o[3]) : "memory");
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(KF + ks));
            if (!__all_sync(0xffffffffu, tile_wait(bar(VE + ks), free_ph, &abort_flag))) { fail(); ok = false; break; }
            // V: a lane takes the words 2 p, 2 p + 1 of a channel
#pragma unroll 4
            for (int it = 0; it < D / 32; ++it) {
                const int ch = 32 * it + 8 * dw + sub;
                uint32_t w0, w1, sh, sc, o[4];
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w0), "=r"(w1) : "r"(raw + P::HALF + P::K_CODES + ch * 32 + p * 8));
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sh) : "r"(raw + P::HALF + P::K_SHIFTS + 4 * ch));
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(sc) : "r"(raw + P::HALF + P::K_SCALES + ch));
                const uint32_t y = shifts_of_unit(sh, 2 * p), s2 = scale_pair(sc), dst = v_t + ch * 128;
                hif4_word_values(w0, y, s2, o);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + ((uint32_t)((2 * p) ^ (ch & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                             "r"(o[2]), "r"(o[3]) : "memory");
                hif4_word_values(w1, y >> 2, s2, o);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + ((uint32_t)((2 * p + 1) ^ (ch & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                             "r"(o[2]), "r"(o[3]) : "memory");
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) { mbar_arrive(bar(VF + ks)); mbar_arrive(bar(RE + rs)); }
        }
    } else if (warp < C::W_LD) {
        // ------------------------------------------------------------------ MMAs of a tile
        const int h = warp - C::W_MMA;
        if (n > 0 && elect_one()) {
            constexpr uint32_t ID_S = umma_idesc_bf16(128, 64), ID_O = umma_idesc_bf16(128, D);
            bool good = tile_wait(bar(QF), 0, &abort_flag);
            tc_fence_after();
            const int behind = alt ? 2 : 1;                          // O += P V of a page goes behind the tile's next S
#pragma unroll 1
            for (int j = 0; j < n + behind && good; ++j) {
                if (j < n) {                                         // S of page j, the tile's page jj
                    const bool mine = alt ? (j & 1) == h : h < tiles;
                    const int jj = alt ? j >> 1 : j;
                    good = tile_wait(bar(KF + j % C::KS), (uint32_t)(j / C::KS) & 1u, &abort_flag) &&
                           (!mine || jj == 0 || tile_wait(bar(SR + h), (uint32_t)(jj - 1) & 1u, &abort_flag));
                    if (!good) break;
                    tc_fence_after();
                    if (mine) {
                        const uint32_t kl = umma_desc_lo(smem + (j % C::KS) * C::K_STAGE), d = tmem + C::S_COL + 64 * h;
#pragma unroll
                        for (int term = 0; term < C::TERMS; ++term) {
                            const int i = h * C::TERMS + term;
                            const uint32_t qt = tmem + C::Q_COL + i * (D / 2), ql = umma_desc_lo(smem + C::Q_OFF + (i - C::Q_FIT) * C::Q_TERM);
                            if (i < C::Q_FIT) {
#pragma unroll
                                for (int k = 0; k < D / 16; ++k)
                                    umma_bf16_ts_lo(d, qt + 8 * k, kl + (k / 4) * (8192 >> 4) + (k % 4) * 2, ID_S, term + k > 0);
                            } else {
#pragma unroll
                                for (int k = 0; k < D / 16; ++k)
                                    umma_bf16_ss_lo(d, ql + (k / 4) * (16384 >> 4) + (k % 4) * 2, kl + (k / 4) * (8192 >> 4) + (k % 4) * 2, ID_S,
                                                    term + k > 0);
                            }
                        }
                        umma_commit(bar(SF + h));
                        umma_commit(bar(KE + j % C::KS));
                    } else {
                        mbar_arrive(bar(KE + j % C::KS));            // a page that is not this tile's
                    }
                }
                if (j >= behind) {                                   // O += P V of page i
                    const int i = j - behind, ii = alt ? i >> 1 : i;
                    const bool mine = alt ? (i & 1) == h : h < tiles;
                    good = tile_wait(bar(VF + i % C::KS), (uint32_t)(i / C::KS) & 1u, &abort_flag) &&
                           (!mine || tile_wait(bar(PF + h), (uint32_t)ii & 1u, &abort_flag));
                    if (!good) break;
                    tc_fence_after();
                    if (mine) {
                        const uint32_t vl = umma_desc_lo(smem + C::V_OFF + (i % C::KS) * C::V_STAGE);
#pragma unroll
                        for (int term = 0; term < C::TERMS; ++term)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_bf16_ts_lo(tmem + h * D, tmem + C::P_COL + C::P_COLS * h + term * 32 + 8 * k, vl + 2 * k, ID_O,
                                                ii > 0 || term + k > 0);
                        umma_commit(bar(OD + h));
                        umma_commit(bar(VE + i % C::KS));
                    } else {
                        mbar_arrive(bar(VE + i % C::KS));
                    }
                }
            }
            // Every commit has arrived before this shared memory goes to another CTA, and this tile's O is complete.  The stages of the last
            // pages are not enough for that: with both tiles on the same rows the last page is one tile's and the other has only
            // arrived for it, while its own last product may still run.
            for (int i = max(n - C::KS, 0); i < n && good; ++i)
                good = tile_wait(bar(KE + i % C::KS), (uint32_t)(i / C::KS) & 1u, &abort_flag) &&
                       tile_wait(bar(VE + i % C::KS), (uint32_t)(i / C::KS) & 1u, &abort_flag);
            const int own = alt ? (n + 1 - h) >> 1 : h < tiles ? n : 0;      // pages of this tile
            if (good && own > 0) good = tile_wait(bar(OD + h), (uint32_t)(own - 1) & 1u, &abort_flag);
            if (!good) { fail(); ok = false; }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ loads
        int ids = -1;
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            if (SELFTEST && blockIdx.x == 0 && j == 2) break;
            if ((j & 31) == 0) ids = j + lane < n ? c.page(b, j0 + j + lane) : -1;
            const int id = __shfl_sync(0xffffffffu, ids, j & 31), rs = j % C::RS;
            if (!__all_sync(0xffffffffu, tile_wait(bar(RE + rs), (uint32_t)(j / C::RS + 1) & 1u, &abort_flag))) { fail(); ok = false; break; }
            if (lane == 0) {
                there[j & 15] = id >= 0;
                if (id >= 0) {
                    mbar_expect_tx(bar(RF + rs), P::BYTES);
                    bulk_load(smem + C::RAW_OFF + rs * P::BYTES, c.pages + ((long long)id * c.Hkv + kv) * P::BYTES, P::BYTES, bar(RF + rs));
                } else {
                    mbar_arrive(bar(RF + rs));                       // the page's tokens are left out; whatever is here has finite values
                    c.invalid();
                }
            }
            __syncwarp();
        }
    }
    if (!ok) let_copies_land();
    tc_fence_before();
    __syncthreads();                                                 // every product is complete (each issuer waited for its tile's last one)
    tc_fence_after();
    const bool good = abort_flag == 0;
    const uint32_t t_o = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (h_sm & 1) * D;
    // O of the other tile, its reference and sum: [d + 2][128] floats over the K and V tiles
    float* const other = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)));
    if (alt) {
        if (good && warp < C::SMW && h_sm == 1) {
            other[D * 128 + r] = m;
            other[(D + 1) * 128 + r] = l;
            if (n_tile > 0) {
#pragma unroll 1
                for (int y = 0; y < D; y += 32) {
                    uint32_t o[32];
                    tmem_ld32(t_o + y, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) other[(y + i) * 128 + r] = __uint_as_float(o[i]);
                }
            }
        }
        __syncthreads();
    }
    if (good && warp < (alt ? 4 : 4 * tiles)) {
        float f0 = 1.f, f1 = 0.f;
        if (alt) {
            const float m1 = other[D * 128 + r], M = fmaxf(m, m1);
            f0 = m == -INFINITY ? 0.f : ex2_approx(m - M);
            f1 = m1 == -INFINITY ? 0.f : ex2_approx(m1 - M);
            l = l * f0 + other[(D + 1) * 128 + r] * f1;
            m = M;
        }
        const float inv = splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
        const long long part = ((long long)slot * C::QT + h_sm) * a.splits + sp;
#pragma unroll 1
        for (int y = 0; y < D; y += 32) {
            uint32_t o[32];
            if (n_tile > 0) {
                tmem_ld32(t_o + y, o);
                tmem_wait_ld();
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0;
            }
            if (alt && n > 1) {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + other[(y + i) * 128 + r] * f1);
            }
            if (!have) continue;
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * inv);
            if (splits == 1) {
                tile_store32(a, (((long long)b * a.Hq + head) * a.N + tok) * D + y, o);
            } else {
                uint4* dst = reinterpret_cast<uint4*>(a.part_o + (part * 128 + r) * D + y);
#pragma unroll
                for (int i = 0; i < 8; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
        }
        if (splits > 1 && have) a.part_ml[part * 128 + r] = make_float2(m, l);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == C::W_MMA) tmem_dealloc(tmem, 512);
}

// Joins the splits: a warp per row.
template <int D>
__global__ void __launch_bounds__(256)
cache_attention_join_kernel(const __grid_constant__ TileArgs a, int QT)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const long long row_id = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int r = (int)(row_id % (128 * QT)), slot = (int)(row_id / (128 * QT));
    int w = a.full + slot;
    const int item = a.items - 1 - w % a.items; w /= a.items;
    const int kv = w % a.cache.Hkv, b = w / a.cache.Hkv;
    const int first = a.units.first[kv], rows = (a.units.first[kv + 1] - first) * a.N, row = item * 128 * QT + r;
    if (row >= rows) return;
    const int head = a.units.head[first + row / a.N], tok = row % a.N;
    const long long p0 = ((long long)slot * QT + r / 128) * a.splits;
    const int rr = r % 128;
    float M = -INFINITY, L = 0.f, o[D / 32];
    for (int x = 0; x < a.splits; ++x) M = fmaxf(M, a.part_ml[(p0 + x) * 128 + rr].x);
#pragma unroll
    for (int y = 0; y < D / 32; ++y) o[y] = 0.f;
#pragma unroll 4
    for (int x = 0; x < a.splits; ++x) {
        const float2 ml = a.part_ml[(p0 + x) * 128 + rr];
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        L = fmaf(ml.y, f, L);
        const float* src = a.part_o + ((p0 + x) * 128 + rr) * D + 2 * lane;
#pragma unroll
        for (int y = 0; y < D / 64; ++y) {
            const float2 v = *reinterpret_cast<const float2*>(src + 64 * y);
            o[2 * y] = fmaf(v.x, f, o[2 * y]);
            o[2 * y + 1] = fmaf(v.y, f, o[2 * y + 1]);
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const long long at = (((long long)b * a.Hq + head) * a.N + tok) * D + 2 * lane;
#pragma unroll
    for (int y = 0; y < D / 64; ++y) tile_store(a, at + 64 * y, o[2 * y] * inv, o[2 * y + 1] * inv);
}

template <typename T, int D, bool SELFTEST = false>
static cudaError_t tile_d(const TileArgs& a, cudaStream_t st)
{
    using C = TileCfg<D, __is_same(T, __half)>;
    static SmemOptIn opt;
    if (!opt.ensure(cache_attention_kernel<T, D, SELFTEST>, C::SMEM)) return cudaErrorInvalidValue;
    const unsigned blocks = (unsigned)(a.cache.B * a.cache.Hkv * a.items), split = blocks - (unsigned)a.full;
    const cudaError_t e = launch_dependent(cache_attention_kernel<T, D, SELFTEST>, (unsigned)a.full + split * (unsigned)a.splits, C::THREADS, C::SMEM, st, a);
    if (e != cudaSuccess || split == 0) return e;
    return launch_dependent(cache_attention_join_kernel<D>, split * (16 * C::QT), 256, 0, st, a, C::QT);
}

int attention_tile_rows(int dtype, int d) { return 128 * (d == 64 || (d == 128 && dtype == HIFA4_BF16) ? 2 : 1); }

cudaError_t launch_cache_attention(int dtype, int d, const TileArgs& a, cudaStream_t st)
{
    const bool bf = dtype == HIFA4_BF16;
    switch (d) {
    case 64: return bf ? tile_d<__nv_bfloat16, 64>(a, st) : tile_d<__half, 64>(a, st);
    case 128: return bf ? tile_d<__nv_bfloat16, 128>(a, st) : tile_d<__half, 128>(a, st);
    default: return bf ? tile_d<__nv_bfloat16, 256>(a, st) : tile_d<__half, 256>(a, st);
    }
}

cudaError_t launch_cache_attention_selftest(const TileArgs& a, cudaStream_t st) { return tile_d<__nv_bfloat16, 128, true>(a, st); }

}  // namespace hifa4
