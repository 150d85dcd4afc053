// Paged HIF4 cache: quantization of new tokens into pages, and the way back to their values.
#include "hifa4_cache.cuh"

namespace hifa4 {

// Nibbles 8 + m of a subgroup's four codes in the low 16 bits, element i in nibble i (above them: anything).  k: the shift.  As
// hif4_unit_values, with 8 more in the low bits of the magic constant: the low bits of y are 8 + m, and no carry leaves a nibble when
// y's multiples by powers of 16 are added up (three instructions for four codes; gathered as bytes and then as nibbles it takes six,
// and 32K tokens 51 us instead of 48).
__device__ __forceinline__ uint32_t subgroup_nibbles(const float* x, int k, const Hif4Group& g)
{
    const float magic = __uint_as_float(0x4B400008u + ((uint32_t)k << 23));
    const uint64_t mm = pack2(magic, magic);
    float y0, y1, y2, y3;
    unpack2(add2(mul2_rz(pack2(x[0], x[1]), g.inv44), mm), y0, y1);
    unpack2(add2(mul2_rz(pack2(x[2], x[3]), g.inv44), mm), y2, y3);
    return __float_as_uint(y3) * 4096 + (__float_as_uint(y2) * 256 + (__float_as_uint(y1) * 16 + __float_as_uint(y0)));
}

// The larger magnitudes of packed pairs, of either sign.
template <typename T, bool NAN_WINS> __device__ __forceinline__ uint32_t max_mag(uint32_t a, uint32_t b)
{
    uint32_t r;
    if constexpr (__is_same(T, __half)) {
        if (NAN_WINS) asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    } else {
        if (NAN_WINS) asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    }
    return r;
}

// Largest magnitude of a group, of which each of four lanes has 16 values (packed pairs).  NAN_WINS: a NaN if there is one, else
// NaN are passed over.
template <typename T, bool NAN_WINS> __device__ __forceinline__ float group_max(const uint32_t (&x)[8])
{
    auto max2 = [](uint32_t a, uint32_t b) { return NAN_WINS ? max16_nan<T>(a, b) : max16<T>(a, b); };
    uint32_t m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = max_mag<T, NAN_WINS>(x[i], x[i + 4]);
    m[0] = abs16<T>(max_mag<T, NAN_WINS>(max_mag<T, NAN_WINS>(m[0], m[1]), max_mag<T, NAN_WINS>(m[2], m[3])));
    m[0] = max2(m[0], __shfl_xor_sync(0xffffffffu, m[0], 1));
    m[0] = max2(m[0], __shfl_xor_sync(0xffffffffu, m[0], 2));
    m[0] = max2(m[0], __byte_perm(m[0], m[0], 0x1032));
    float a, b;
    Pair16<T>::unpack(m[0], a, b);
    return a;
}

// A lane's 16 consecutive values (two units) of a group: nibbles of the four subgroups (subgroup_nibbles) and their shifts.
// GENERAL: what lies above the E6M2 range saturates, a NaN becomes zero; otherwise there are none.
template <typename T, bool GENERAL>
__device__ __forceinline__ void quantize16(const uint32_t (&xw)[8], const Hif4Group& g, uint32_t (&nib)[4], int (&k)[4])
{
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) Pair16<T>::unpack(xw[4 * u + i], x[2 * i], x[2 * i + 1]);
        if (GENERAL) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -g.top), g.top) : 0.f;
        }
        const float a0 = fmaxf(max3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2])), fabsf(x[3]));
        const float a1 = fmaxf(max3(fabsf(x[4]), fabsf(x[5]), fabsf(x[6])), fabsf(x[7]));
        const int n0 = max((int)__float_as_uint(a0) + g.tadd, 0) >> 23, n1 = max((int)__float_as_uint(a1) + g.tadd, 0) >> 23;
        const int a = (n0 + n1 + 2) >> 2;                                    // (see hif4_unit)
        k[2 * u] = max(n0, a);
        k[2 * u + 1] = max(n1, a);
        nib[2 * u] = subgroup_nibbles(x, k[2 * u], g);
        nib[2 * u + 1] = subgroup_nibbles(x + 4, k[2 * u + 1], g);
    }
}
// The same from the values alone; *code: the group's scale.  Whole warp: the general form runs where a group of the warp needs it.
template <typename T> __device__ __forceinline__ void quantize_group(const uint32_t (&xw)[8], uint32_t (&nib)[4], int (&k)[4], int* code)
{
    const float A = group_max<T, true>(xw);
    Hif4Group g = hif4_group(A);
    if (__any_sync(0xffffffffu, !(A <= g.top))) {
        float B = group_max<T, false>(xw);
        g = hif4_group(B == B ? B : 0.f);                                    // (only NaN: zeros)
        quantize16<T, true>(xw, g, nib, k);
    } else {
        quantize16<T, false>(xw, g, nib, k);
    }
    *code = g.code;
}

// One CTA per (sequence, KV head, page that the new tokens touch); four lanes per 64-element group, 16 elements each, which
// are whole words of the page's layout.  K: rows straight from global memory.  V: the page's rows, old ones from the tail and new
// ones, turned in shared memory; a team takes two adjacent channels.
// The CTA of a sequence's first page is the one that reads the old tail, so it also writes the new one.
template <typename T, int D>
__global__ void __launch_bounds__(256)
cache_append_kernel(const CacheView c, int n, const int* __restrict__ n_new, const uint16_t* __restrict__ k, Strides ks,
                    const uint16_t* __restrict__ v, Strides vs, const float* __restrict__ inv_s)
{
    using P = Page<D>;
    constexpr int NG = P::NG, CH = D / 8, KT = 64 * NG * 4 / 256, VT = 64 * CH / 256;
    __shared__ __align__(16) uint4 rows[64 * CH];        // 16-byte chunk i of row r at i ^ (r / 16): the four lanes of a team read
                                                         // rows 16 apart
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.y / c.Hkv, h = blockIdx.y % c.Hkv, tid = threadIdx.x;
    const int len = c.len(b), cnt = n_new ? __ldg(n_new + b) : n;
    const int slot = c.slots ? __ldg(c.slots + b) : b;
    if (len < 0 || cnt < 0 || cnt > n || cnt > len || slot < 0 || slot >= c.n_tails) {
        if (blockIdx.x == 0 && tid == 0) c.invalid();
        return;
    }
    if (cnt == 0) return;
    const int begin = len - cnt, p = (begin >> 6) + (int)blockIdx.x, last = (len - 1) >> 6;
    if (p > last) return;
    const int page = c.page(b, p);
    uint4* tail = reinterpret_cast<uint4*>(c.v_tail + ((long long)slot * c.Hkv + h) * 64 * D);
    const int lo = max(begin - 64 * p, 0), hi = min(len - 64 * p, 64);     // the page's rows [lo, hi) are new
    const uint16_t* kb = k + b * ks.b + h * ks.h + (64ll * p - begin) * ks.t;   // row 0 of the page
    const uint16_t* vb = v + b * vs.b + h * vs.h + (64ll * p - begin) * vs.t;
    uint4 vx[VT], kx[KT][2];
#pragma unroll
    for (int i = 0; i < VT; ++i) {
        const int r = (i * 256 + tid) / CH, ch = (i * 256 + tid) % CH;
        vx[i] = make_uint4(0, 0, 0, 0);
        if (r < lo) vx[i] = tail[r * CH + ch];
        else if (r < hi) vx[i] = __ldg(reinterpret_cast<const uint4*>(vb + r * vs.t) + ch);
    }
    // K: task = (row, group, lane of the team)
#pragma unroll
    for (int i = 0; i < KT; ++i) {
        const int t = i * 256 + tid, r = t / (4 * NG);
        kx[i][0] = kx[i][1] = make_uint4(0, 0, 0, 0);
        if (r >= lo && r < hi) {
            const uint4* src = reinterpret_cast<const uint4*>(kb + r * ks.t + t % (4 * NG) / 4 * 64 + t % 4 * 16);
            kx[i][0] = __ldg(src);
            kx[i][1] = __ldg(src + 1);
        }
    }
#pragma unroll
    for (int i = 0; i < VT; ++i) {
        const int r = (i * 256 + tid) / CH, ch = (i * 256 + tid) % CH;
        rows[r * CH + (ch ^ (r >> 4))] = vx[i];
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        // New rows that the last page may be continued from: all of an incomplete page; of a page that was begun before and is full now,
        // all but the last, which any append behind a cut inside the page brings itself (drafted tokens that are taken back).
        const int used = len - 64 * last, t0 = last == p ? lo : 0, t1 = used < 64 ? used : t0 > 0 ? 63 : 0;
        const uint16_t* vl = v + b * vs.b + h * vs.h + (64ll * last - begin) * vs.t;
        for (int i = tid + t0 * CH; i < t1 * CH; i += 256) tail[i] = __ldg(reinterpret_cast<const uint4*>(vl + i / CH * vs.t) + i % CH);
    }
    if (page < 0) {
        if (tid == 0) c.invalid();
        return;
    }
    uint8_t* pg = c.pages + ((long long)page * c.Hkv + h) * P::BYTES;
#pragma unroll
    for (int i = 0; i < KT; ++i) {
        const int t = i * 256 + tid, r = t / (4 * NG), G = t % (4 * NG) / 4, j = t % 4;
        const bool in = r >= lo && r < hi;
        if (!__any_sync(0xffffffffu, in)) continue;
        uint32_t xw[8] = {kx[i][0].x, kx[i][0].y, kx[i][0].z, kx[i][0].w, kx[i][1].x, kx[i][1].y, kx[i][1].z, kx[i][1].w};
        if (inv_s) {                                                         // FP32 product, rounded once to the activation dtype
            const float4* f = reinterpret_cast<const float4*>(inv_s + h * D + 64 * G + 16 * j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 fe = __ldg(f + e);
                float x0, x1;
                Pair16<T>::unpack(xw[2 * e], x0, x1);
                xw[2 * e] = Pair16<T>::round_pack(x0 * fe.x, x1 * fe.y);
                Pair16<T>::unpack(xw[2 * e + 1], x0, x1);
                xw[2 * e + 1] = Pair16<T>::round_pack(x0 * fe.z, x1 * fe.w);
            }
        }
        uint32_t nib[4];
        int sh[4], code;
        quantize_group<T>(xw, nib, sh, &code);
        uint32_t s = (uint32_t)(sh[0] | sh[1] << 16 | sh[2] << 2 | sh[3] << 18) << (4 * j);
        s |= __shfl_xor_sync(0xffffffffu, s, 1);
        s |= __shfl_xor_sync(0xffffffffu, s, 2);
        if (!in) continue;
        *reinterpret_cast<uint2*>(pg + P::K_CODES + r * (D / 2) + j * 8 * NG + 8 * G) =
            make_uint2(__byte_perm(nib[0], nib[1], 0x5410), __byte_perm(nib[2], nib[3], 0x5410));
        if (j == 0) {
            *reinterpret_cast<uint32_t*>(pg + P::K_SHIFTS + 4 * (r * NG + G)) = s;
            pg[P::K_SCALES + r * NG + G] = (uint8_t)code;
        }
    }
    uint8_t* vp = pg + P::HALF;
    const uint32_t* words = reinterpret_cast<const uint32_t*>(rows);
#pragma unroll
    for (int t = tid; t < D * 2; t += 256) {                                 // task = (pair of channels, lane of the team)
        const int cp = t / 4, j = t % 4;
        uint32_t xa[8], xb[8];                                               // channels 2 cp and 2 cp + 1, pairs of tokens
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t x0, x1;
            {
                const int r = 16 * j + 2 * e;
                x0 = words[(r * CH + ((cp / 4) ^ j)) * 4 + cp % 4];
                x1 = words[((r + 1) * CH + ((cp / 4) ^ j)) * 4 + cp % 4];
            }
            xa[e] = __byte_perm(x0, x1, 0x5410);
            xb[e] = __byte_perm(x0, x1, 0x7632);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t (&xw)[8] = x ? xb : xa;
            uint32_t nib[4];
            int sh[4], code;
            quantize_group<T>(xw, nib, sh, &code);                             // subgroups: tokens 16 j + 4 i + (0..3); word h: i = h and h + 2
            uint32_t s = (uint32_t)(sh[0] | sh[1] << 2 | sh[2] << 16 | sh[3] << 18) << (4 * j);
            s |= __shfl_xor_sync(0xffffffffu, s, 1);
            s |= __shfl_xor_sync(0xffffffffu, s, 2);
            const int ch = 2 * cp + x;
            *reinterpret_cast<uint2*>(vp + P::K_CODES + ch * 32 + j * 8) =
                make_uint2(__byte_perm(nib[0], nib[2], 0x5410), __byte_perm(nib[1], nib[3], 0x5410));
            if (j == 0) {
                *reinterpret_cast<uint32_t*>(vp + P::K_SHIFTS + 4 * ch) = s;
                vp[P::K_SCALES + ch] = (uint8_t)code;
            }
        }
    }
}

// Eight values of a row from their BF16 pairs.
__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint32_t (&x)[4]) { *reinterpret_cast<uint4*>(p) = make_uint4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store8(float* p, const uint32_t (&x)[4])
{
    reinterpret_cast<uint4*>(p)[0] = make_uint4(x[0] << 16, x[0] & 0xFFFF0000u, x[1] << 16, x[1] & 0xFFFF0000u);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(x[2] << 16, x[2] & 0xFFFF0000u, x[3] << 16, x[3] & 0xFFFF0000u);
}

// Two CTAs per (sequence, KV head, page), one for K and one for V; both straight from global memory (32K tokens of 8 heads, d = 128: 27
// us, the copy rate; by way of shared memory in one CTA 38).  K: a thread per unit of a row.  V: a thread per word of eight
// channels, whose 64 values are turned in registers, so that it stores 16 bytes (FP32: 32) of eight rows; a warp has four words of
// 64 channels and stores whole 128-byte lines (eight words of 32 channels: 32 us).
template <typename O, int D>
__global__ void __launch_bounds__(128, 10)
cache_read_kernel(const CacheView c, int n, const int* __restrict__ start, O* __restrict__ k_out, O* __restrict__ v_out)
{
    using P = Page<D>;
    constexpr int NG = P::NG, AHEAD = 4;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.y / c.Hkv, h = blockIdx.y % c.Hkv, tid = threadIdx.x + 128 * blockIdx.z;   // from 128: V
    const int len = c.len(b), begin = start ? __ldg(start + b) : 0;
    if (len < 0 || begin < 0) {
        if (blockIdx.x == 0 && tid == 0) c.invalid();
        return;
    }
    const int p = (begin >> 6) + (int)blockIdx.x;
    const int end = (int)min((long long)len, (long long)begin + n);
    if (64ll * p >= end) return;
    const int page = c.page(b, p);
    if (page < 0) {
        if (tid == 0) c.invalid();
        return;
    }
    const uint8_t* pg = c.pages + ((long long)page * c.Hkv + h) * P::BYTES;
    const int lo = max(begin - 64 * p, 0), hi = min(end - 64 * p, 64);
    const long long row0 = ((long long)b * c.Hkv + h) * n + 64ll * p - begin;
    if (tid < 128) {
        const int u = tid % (D / 8), G = u / 8, uu = u % 8;
        constexpr int ROWS = 128 / (D / 8);                      // rows at a time
#pragma unroll 1
        for (int r0 = tid / (D / 8); r0 < 64; r0 += ROWS * AHEAD) {
            uint32_t w[AHEAD], sh[AHEAD], sc[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int r = r0 + i * ROWS;
                if (r < lo || r >= hi) continue;
                w[i] = __ldg(reinterpret_cast<const uint32_t*>(pg + P::K_CODES + r * (D / 2) + (uu / 2) * 8 * NG + 8 * G + uu % 2 * 4));
                sh[i] = __ldg(reinterpret_cast<const uint32_t*>(pg + P::K_SHIFTS + 4 * (r * NG + G)));
                sc[i] = __ldg(pg + P::K_SCALES + r * NG + G);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int r = r0 + i * ROWS;
                if (r < lo || r >= hi) continue;
                uint32_t x[4];
                hif4_word_values(w[i], shifts_of_unit(sh[i], uu), scale_pair(sc[i]), x);
                const uint32_t y[4] = {__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410), __byte_perm(x[0], x[1], 0x7632),
                                       __byte_perm(x[2], x[3], 0x7632)};
                store8(k_out + (row0 + r) * D + 8 * u, y);
            }
        }
        return;
    }
    const uint8_t* vp = pg + P::HALF;
#pragma unroll 1
    for (int t = tid - 128; t < D; t += 128) {
        const int o = t / 4 % (D / 8), w = t % 4 + t / 4 / (D / 8) * 4;
        uint32_t code[8], sh[8], x[8][4];                        // channel 8 o + i: pairs of tokens 16 (w / 2) + 4 (w % 2) + e, + 8
#pragma unroll
        for (int i = 0; i < 8; ++i) code[i] = __ldg(reinterpret_cast<const uint32_t*>(vp + P::K_CODES + (8 * o + i) * 32 + w * 4));
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const uint4 y = __ldg(reinterpret_cast<const uint4*>(vp + P::K_SHIFTS + 32 * o) + i / 4);
            sh[i] = y.x; sh[i + 1] = y.y; sh[i + 2] = y.z; sh[i + 3] = y.w;
        }
        const uint2 sc = __ldg(reinterpret_cast<const uint2*>(vp + P::K_SCALES + 8 * o));
#pragma unroll
        for (int i = 0; i < 8; ++i)
            hif4_word_values(code[i], shifts_of_unit(sh[i], w), scale_pair((i < 4 ? sc.x : sc.y) >> 8 * (i % 4) & 255), x[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int r = 16 * (w / 2) + 4 * (w % 2) + e % 4 + e / 4 * 8;
            if (r < lo || r >= hi) continue;
            const uint32_t sel = e < 4 ? 0x5410 : 0x7632;
            const uint32_t y[4] = {__byte_perm(x[0][e % 4], x[1][e % 4], sel), __byte_perm(x[2][e % 4], x[3][e % 4], sel),
                                   __byte_perm(x[4][e % 4], x[5][e % 4], sel), __byte_perm(x[6][e % 4], x[7][e % 4], sel)};
            store8(v_out + (row0 + r) * D + 8 * o, y);
        }
    }
}

template <typename T, int D>
static cudaError_t append_d(const CacheView& c, int n, const int* n_new, const void* k, Strides ks, const void* v, Strides vs,
                            const float* inv_s, cudaStream_t st)
{
    return launch_dependent(cache_append_kernel<T, D>, dim3((unsigned)((n + 126ll) / 64), (unsigned)(c.B * c.Hkv)), 256, 0, st, c, n, n_new,
                            (const uint16_t*)k, ks, (const uint16_t*)v, vs, inv_s);
}

cudaError_t launch_cache_append(int dtype, int d, const CacheView& c, int n, const int* n_new, const void* k, Strides ks,
                                const void* v, Strides vs, const float* inv_s, cudaStream_t st)
{
    const bool bf = dtype == HIFA4_BF16;
    switch (d) {
    case 64: return bf ? append_d<__nv_bfloat16, 64>(c, n, n_new, k, ks, v, vs, inv_s, st) : append_d<__half, 64>(c, n, n_new, k, ks, v, vs, inv_s, st);
    case 128: return bf ? append_d<__nv_bfloat16, 128>(c, n, n_new, k, ks, v, vs, inv_s, st) : append_d<__half, 128>(c, n, n_new, k, ks, v, vs, inv_s, st);
    default: return bf ? append_d<__nv_bfloat16, 256>(c, n, n_new, k, ks, v, vs, inv_s, st) : append_d<__half, 256>(c, n, n_new, k, ks, v, vs, inv_s, st);
    }
}

template <typename O, int D>
static cudaError_t read_d(const CacheView& c, int n, const int* start, void* k, void* v, cudaStream_t st)
{
    return launch_dependent(cache_read_kernel<O, D>, dim3((unsigned)((n + 126ll) / 64), (unsigned)(c.B * c.Hkv), 2), 128, 0, st, c, n, start, (O*)k, (O*)v);
}

cudaError_t launch_cache_read(int d, const CacheView& c, int n, const int* start, int out_dtype, void* k, void* v, cudaStream_t st)
{
    const bool bf = out_dtype == HIFA4_BF16;
    switch (d) {
    case 64: return bf ? read_d<__nv_bfloat16, 64>(c, n, start, k, v, st) : read_d<float, 64>(c, n, start, k, v, st);
    case 128: return bf ? read_d<__nv_bfloat16, 128>(c, n, start, k, v, st) : read_d<float, 128>(c, n, start, k, v, st);
    default: return bf ? read_d<__nv_bfloat16, 256>(c, n, start, k, v, st) : read_d<float, 256>(c, n, start, k, v, st);
    }
}

}  // namespace hifa4
