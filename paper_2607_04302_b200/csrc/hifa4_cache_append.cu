// Paged HIF4 cache: quantization of new tokens into pages, and the way back to their values.
#include "hifa4_cache.cuh"

namespace hifa4 {

// Packed nibbles 8 + m of four biased quotients (hif4_unit: the low byte of bits(y) is the signed code m).
__device__ __forceinline__ uint32_t nibbles4(const float* y)
{
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((__float_as_uint(y[e]) + 8u) & 15u) << (4 * e);
    return w;
}

// One unit (8 elements) of a group: clamps what lies above the E6M2 range, drops NaN, and returns codes and shifts.
__device__ __forceinline__ void quantize_unit(float (&x)[8], const Hif4Group& g, float (&y)[8], int& k0, int& k1)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] > g.top ? g.top : x[i] < -g.top ? -g.top : x[i] == x[i] ? x[i] : 0.f;
    const float a0 = fmaxf(max3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2])), fabsf(x[3]));
    const float a1 = fmaxf(max3(fabsf(x[4]), fabsf(x[5]), fabsf(x[6])), fabsf(x[7]));
    uint32_t w[4];
    int a;
    hif4_unit(x, a0, a1, g, w, y, a, k0, k1);
}

// One CTA per (sequence, KV head, page that the new tokens touch).  K: a thread per 64-element group of a row.  V: the
// page's rows, old ones from the tail and new ones, gathered in shared memory; a thread per channel.
// The CTA of a sequence's first page is the one that reads the old tail, so it also writes the new one.
template <typename T, int D>
__global__ void __launch_bounds__(256)
cache_append_kernel(const CacheView c, int n, const int* __restrict__ n_new, const uint16_t* __restrict__ k, Strides ks,
                    const uint16_t* __restrict__ v, Strides vs, const float* __restrict__ inv_s)
{
    using P = Page<D>;
    constexpr int NG = P::NG;
    __shared__ __align__(16) uint16_t rows[64 * D];
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
    uint16_t* tail = c.v_tail + ((long long)slot * c.Hkv + h) * 64 * D;
    const int lo = max(begin - 64 * p, 0), hi = min(len - 64 * p, 64);     // the page's rows [lo, hi) are new
    const uint16_t* kb = k + b * ks.b + h * ks.h + (64ll * p - begin) * ks.t;   // row 0 of the page
    const uint16_t* vb = v + b * vs.b + h * vs.h + (64ll * p - begin) * vs.t;
    for (int i = tid; i < 64 * (D / 8); i += 256) {
        const int r = i / (D / 8), ch = i % (D / 8) * 8;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (r < lo) x = *reinterpret_cast<const uint4*>(tail + r * D + ch);
        else if (r < hi) x = __ldg(reinterpret_cast<const uint4*>(vb + r * vs.t + ch));
        *reinterpret_cast<uint4*>(rows + r * D + ch) = x;
    }
    __syncthreads();
    if (blockIdx.x == 0) {                                                   // rows of the incomplete page that are new
        const int t0 = last == p ? lo : 0, t1 = len & 63;
        const uint16_t* vl = v + b * vs.b + h * vs.h + (64ll * last - begin) * vs.t;
        for (int i = tid; i < t1 * (D / 8); i += 256) {
            const int r = i / (D / 8), ch = i % (D / 8) * 8;
            if (r >= t0) *reinterpret_cast<uint4*>(tail + r * D + ch) = __ldg(reinterpret_cast<const uint4*>(vl + r * vs.t + ch));
        }
    }
    if (page < 0) {
        if (tid == 0) c.invalid();
        return;
    }
    uint8_t* pg = c.pages + ((long long)page * c.Hkv + h) * P::BYTES;
    for (int i = tid + lo * NG; i < hi * NG; i += 256) {
        const int r = i / NG, G = i % NG;
        const uint4* src = reinterpret_cast<const uint4*>(kb + r * ks.t + 64 * G);
        uint32_t xw[32];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint4 x = __ldg(src + j);
            xw[4 * j] = x.x; xw[4 * j + 1] = x.y; xw[4 * j + 2] = x.z; xw[4 * j + 3] = x.w;
        }
        float A = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float x0, x1;
            Pair16<T>::unpack(xw[j], x0, x1);
            if (inv_s) {                                                     // FP32 product, rounded once to the activation dtype
                const float2 f = __ldg(reinterpret_cast<const float2*>(inv_s + h * D + 64 * G) + j);
                xw[j] = Pair16<T>::round_pack(x0 * f.x, x1 * f.y);
                Pair16<T>::unpack(xw[j], x0, x1);
            }
            A = max3(A, fabsf(x0), fabsf(x1));
        }
        const Hif4Group g = hif4_group(A);
        uint32_t shifts = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            float x[8], y[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) Pair16<T>::unpack(xw[4 * u + j], x[2 * j], x[2 * j + 1]);
            int k0, k1;
            quantize_unit(x, g, y, k0, k1);
            *reinterpret_cast<uint32_t*>(pg + P::K_CODES + r * (D / 2) + (u / 2) * 8 * NG + G * 8 + (u % 2) * 4) =
                nibbles4(y) | nibbles4(y + 4) << 16;
            shifts |= (uint32_t)k0 << (2 * u) | (uint32_t)k1 << (16 + 2 * u);
        }
        *reinterpret_cast<uint32_t*>(pg + P::K_SHIFTS + 4 * i) = shifts;
        pg[P::K_SCALES + i] = (uint8_t)g.code;
    }
    uint8_t* vp = pg + P::HALF;
    for (int ch = tid; ch < D; ch += 256) {
        float A = 0.f;
#pragma unroll 16
        for (int t = 0; t < 64; ++t) A = fmaxf(A, fabsf(In16<T>::to_f(rows[t * D + ch])));
        const Hif4Group g = hif4_group(A);
        uint32_t shifts = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w0 = 0, w1 = 0;
#pragma unroll
            for (int r = 0; r < 2; ++r) {                                    // unit r: tokens 16 i + 8 r + (0..7)
                float x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = In16<T>::to_f(rows[(16 * i + 8 * r + e) * D + ch]);
                int k0, k1;
                quantize_unit(x, g, y, k0, k1);
                w0 |= nibbles4(y) << (16 * r);
                w1 |= nibbles4(y + 4) << (16 * r);
                shifts |= (uint32_t)k0 << (16 * r + 4 * i) | (uint32_t)k1 << (16 * r + 4 * i + 2);
            }
            *reinterpret_cast<uint2*>(vp + P::K_CODES + ch * 32 + i * 8) = make_uint2(w0, w1);
        }
        *reinterpret_cast<uint32_t*>(vp + P::K_SHIFTS + 4 * ch) = shifts;
        vp[P::K_SCALES + ch] = (uint8_t)g.code;
    }
}

__device__ __forceinline__ void store_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }   // exact

// One CTA per (sequence, KV head, page).  A thread per element: bound by its stores.
template <typename O, int D>
__global__ void __launch_bounds__(256)
cache_read_kernel(const CacheView c, int n, const int* __restrict__ start, O* __restrict__ k_out, O* __restrict__ v_out)
{
    using P = Page<D>;
    constexpr int NG = P::NG;
    __shared__ __align__(16) uint32_t sm[P::BYTES / 4];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.y / c.Hkv, h = blockIdx.y % c.Hkv, tid = threadIdx.x;
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
    const uint4* src = reinterpret_cast<const uint4*>(c.pages + ((long long)page * c.Hkv + h) * P::BYTES);
    for (int i = tid; i < P::BYTES / 16; i += 256) reinterpret_cast<uint4*>(sm)[i] = __ldg(src + i);
    __syncthreads();
    const uint8_t* by = reinterpret_cast<const uint8_t*>(sm);
    const int lo = max(begin - 64 * p, 0), hi = min(end - 64 * p, 64);
    const long long row0 = ((long long)b * c.Hkv + h) * n + 64ll * p - begin;
    for (int i = tid; i < 64 * D; i += 256) {
        const int r = i / D, ch = i % D;
        if (r < lo || r >= hi) continue;
        const long long o = (row0 + r) * D + ch;
        {
            const int G = ch / 64, u = ch % 64 / 8, e = ch % 8;
            const uint32_t w = sm[r * (D / 8) + (u / 2) * 2 * NG + 2 * G + u % 2];
            const int sh = (sm[P::K_SHIFTS / 4 + r * NG + G] >> (16 * (e / 4) + 2 * u)) & 3;
            const float s4 = quarter_scale(by[P::K_SCALES + r * NG + G]);
            store_value(k_out + o, (float)(((int)(w >> (4 * e)) & 15) - 8) * __uint_as_float(__float_as_uint(s4) + (sh << 23)));
        }
        {
            const int w_i = 2 * (r / 16) + r / 4 % 2, hf = r / 8 % 2, e = r % 4;
            const uint32_t w = sm[P::HALF / 4 + ch * 8 + w_i];
            const int sh = (sm[(P::HALF + P::K_SHIFTS) / 4 + ch] >> (16 * hf + 2 * w_i)) & 3;
            const float s4 = quarter_scale(by[P::HALF + P::K_SCALES + ch]);
            store_value(v_out + o, (float)(((int)(w >> (16 * hf + 4 * e)) & 15) - 8) * __uint_as_float(__float_as_uint(s4) + (sh << 23)));
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
    return launch_dependent(cache_read_kernel<O, D>, dim3((unsigned)((n + 126ll) / 64), (unsigned)(c.B * c.Hkv)), 256, 0, st, c, n, start, (O*)k, (O*)v);
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
