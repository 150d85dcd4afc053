// C-ABI entry points of the paged HIF4 cache: argument validation, size queries and launches.
#include <cmath>
#include <cstring>

#include "hifa4_cache.cuh"

using namespace hifa4;

namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

bool built(int d) { return d == 64 || d == 128 || d == 256; }

int check_cache(const hifa4_cache* c, bool write)
{
    if (!c || !c->pages || c->n_pages <= 0 || c->Hkv <= 0 || c->Hkv > HIFA4_MAX_HEADS) return HIFA4_ERR_INVALID_ARG;
    if (c->in_dtype != HIFA4_F16 && c->in_dtype != HIFA4_BF16) return HIFA4_ERR_INVALID_ARG;
    if (!built(c->d)) return HIFA4_ERR_UNSUPPORTED;
    if ((uintptr_t)c->pages & 15) return HIFA4_ERR_INVALID_ARG;
    if (write && (!c->v_tail || c->n_tails <= 0 || ((uintptr_t)c->v_tail & 15))) return HIFA4_ERR_INVALID_ARG;
    return HIFA4_OK;
}

int check_seqs(const hifa4_seqs* s, int Hkv)
{
    if (!s || s->B <= 0 || s->max_pages <= 0 || !s->block_table || !s->kv_lens) return HIFA4_ERR_INVALID_ARG;
    if ((long long)s->B * Hkv > 65535 || s->max_pages > (1 << 24)) return HIFA4_ERR_UNSUPPORTED;
    return HIFA4_OK;
}

// A 16-bit tensor [B][H][n][d]: its strides, null where it cannot be read with 16-byte loads.
int check_tensor(const void* p, const hifa4_strides* st, int H, int n, int d, Strides* out)
{
    if (!p || ((uintptr_t)p & 15)) return HIFA4_ERR_INVALID_ARG;
    *out = st ? Strides{st->b, st->h, st->t} : Strides{(long long)H * n * d, (long long)n * d, d};
    if ((out->b | out->h | out->t) & 7) return HIFA4_ERR_INVALID_ARG;
    return HIFA4_OK;
}

// Factors of Smooth-QK, read four at a time; null: none.
bool factors_ok(const float* s) { return !((uintptr_t)s & 15); }

CacheView view(const hifa4_cache* c, const hifa4_seqs* s, int* d_status)
{
    CacheView v;
    std::memset(&v, 0, sizeof(v));
    if (c) {
        v.pages = (uint8_t*)c->pages;
        v.v_tail = (uint16_t*)c->v_tail;
        v.n_pages = c->n_pages;
        v.n_tails = c->n_tails;
        v.Hkv = c->Hkv;
    }
    v.B = s->B;
    v.max_pages = s->max_pages;
    v.table = s->block_table;
    v.lens = s->kv_lens;
    v.slots = s->tail_slots;
    v.d_status = d_status;
    return v;
}

int check_query(const hifa4_cache* c, const hifa4_cache_query* q, CacheUnits* units, int* rows)
{
    if (!q || q->N <= 0) return HIFA4_ERR_INVALID_ARG;
    if (q->out_dtype < HIFA4_F16 || q->out_dtype > HIFA4_F32) return HIFA4_ERR_INVALID_ARG;
    if (q->softmax_scale < 0.f || !std::isfinite(q->softmax_scale)) return HIFA4_ERR_INVALID_ARG;
    if (q->causal != 0 && q->causal != 1) return HIFA4_ERR_INVALID_ARG;
    if (q->N > (1 << 20)) return HIFA4_ERR_UNSUPPORTED;
    HeadMap qmap, kmap;
    const int rc = build_map(q->Hq, c->Hkv, q->q_to_kv, qmap, kmap);
    if (rc) return rc;
    int count[HIFA4_MAX_HEADS + 1] = {0}, most = 0, at = 0;
    for (int h = 0; h < q->Hq; ++h) ++count[qmap.kv_of[h]];
    for (int g = 0; g < c->Hkv; ++g) {
        units->first[g] = (short)at;
        at += count[g];
        most = count[g] > most ? count[g] : most;
        count[g] = units->first[g];                                  // where the head map's next head goes
    }
    for (int h = 0; h < q->Hq; ++h) units->head[count[qmap.kv_of[h]]++] = (uint8_t)h;
    units->first[c->Hkv] = (short)at;
    *rows = most * q->N;
    return HIFA4_OK;
}

struct DecodeLayout {
    int block_rows;
    long long blocks;
    size_t first, part_o, part_ml, begun, seg_ctas, final_ml, page_ml, total;
    DecodeLayout(const hifa4_cache* c, int B, int max_pages, const hifa4_cache_query* q, int rows, bool weight)
    {
        block_rows = decode_block_rows(c->d, rows);
        blocks = (rows + block_rows - 1) / block_rows;
        first = 0;
        size_t off = align256(decode_first_floats(c->d, block_rows) * sizeof(float));
        part_o = off;
        off += align256((size_t)2 * DECODE_CTAS * block_rows * c->d * sizeof(float));
        part_ml = off;
        off += align256((size_t)2 * DECODE_CTAS * block_rows * sizeof(float2));
        begun = off;
        off += align256(DECODE_CTAS * sizeof(int4));
        seg_ctas = off;
        if (weight) off += align256((size_t)B * c->Hkv * blocks * sizeof(int2));
        final_ml = off;
        if (weight) off += align256((size_t)B * q->Hq * sizeof(float2));
        page_ml = off;
        if (weight) off += align256((size_t)B * q->Hq * max_pages * sizeof(float2));
        total = off;
    }
};

// Fills what both kernels' arguments have in common.
template <class Args>
void common_args(Args& a, const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q, const float* s,
                 void* out, int* d_status)
{
    a.cache = view(cache, seqs, d_status);
    a.q = q;
    a.s = s;
    a.Hq = query->Hq;
    a.N = query->N;
    a.causal = query->causal;
    a.out_dtype = query->out_dtype;
    const double scale = query->softmax_scale > 0.f ? query->softmax_scale : 1.0 / std::sqrt((double)cache->d);
    a.scale_log2 = (float)(scale * 1.4426950408889634);
    a.out = out;
}

int check_call(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
               const hifa4_strides* q_strides, const float* s, const void* out, CacheUnits* units, int* rows, Strides* qs)
{
    int rc = check_cache(cache, false);
    if (rc) return rc;
    if ((rc = check_seqs(seqs, cache->Hkv))) return rc;
    if ((rc = check_query(cache, query, units, rows))) return rc;
    if (!out || ((uintptr_t)out & 15) || !factors_ok(s)) return HIFA4_ERR_INVALID_ARG;
    return check_tensor(q, q_strides, query->Hq, query->N, cache->d, qs);
}

int run_decode(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const CacheUnits& units, int rows,
               Strides qs, const void* q, const float* s, void* out, float* lse, const float* weight, float* weight_out,
               void* workspace, size_t workspace_bytes, int* d_status, void* stream, bool selftest = false)
{
    const DecodeLayout lay(cache, seqs->B, seqs->max_pages, query, rows, weight_out != nullptr);
    if (!workspace || workspace_bytes < lay.total || ((uintptr_t)workspace & 255)) return HIFA4_ERR_WORKSPACE;
    if ((2.0 * seqs->max_pages + 1) * seqs->B * cache->Hkv * lay.blocks > 2.0e9) return HIFA4_ERR_UNSUPPORTED;      // steps of work are numbered in 32 bits
    if (weight_out && (long long)seqs->B * ((seqs->max_pages + 63) / 64) > 0x7FFFF000ll) return HIFA4_ERR_UNSUPPORTED;
    const int rc = check_arch();
    if (rc) return rc;
    DecodeArgs a;
    std::memset(&a, 0, sizeof(a));
    common_args(a, cache, seqs, query, q, s, out, d_status);
    char* ws = (char*)workspace;
    a.units = units;
    a.qs = qs;
    a.blocks = (int)lay.blocks;
    a.one = 1;
    a.lse = lse;
    a.weight = weight;
    a.weight_out = weight_out;
    a.first = (float*)(ws + lay.first);
    a.part_o = (float*)(ws + lay.part_o);
    a.part_ml = (float2*)(ws + lay.part_ml);
    a.begun = (int4*)(ws + lay.begun);
    a.seg_ctas = weight_out ? (int2*)(ws + lay.seg_ctas) : nullptr;
    a.final_ml = weight_out ? (float2*)(ws + lay.final_ml) : nullptr;
    a.page_ml = weight_out ? (float2*)(ws + lay.page_ml) : nullptr;
    const cudaError_t e = selftest ? launch_cache_decode_selftest(a, (cudaStream_t)stream)
                                   : launch_cache_decode(cache->in_dtype, cache->d, lay.block_rows, a, (cudaStream_t)stream);
    return e == cudaSuccess ? HIFA4_OK : HIFA4_ERR_CUDA;
}

// The tensor-memory kernel's grid and workspace.  A CTA has an SM to itself; blocks come in waves, and a last wave that does not
// fill the chip takes as long as a full one: the blocks behind the last full wave (or the one before) are split over their pages
// where that shortens the whole.  In units of a page (1 us): a CTA's prologue and epilogue cost 6, joining 6 (four sequences of 5-8K
// tokens, 512 blocks: split in two behind three waves 434 us, in thirteen 507, not split 450; 96 blocks of 1500 tokens
// at most: not split 23, in three 32).
struct TileLayout {
    long long items, blocks, full;
    int splits;
    size_t part_ml, total;
    TileLayout(const hifa4_cache* c, int B, int max_pages, int rows)
    {
        const int block = attention_tile_rows(c->in_dtype, c->d), sms = DECODE_CTAS;
        items = (rows + block - 1) / block;
        blocks = (long long)B * c->Hkv * items;
        full = blocks;
        splits = 1;
        const double fixed = 6.0, pages = max_pages;
        double best = (double)((blocks + sms - 1) / sms) * (pages + fixed);
        for (long long waves = blocks / sms; waves >= 0 && waves >= blocks / sms - 1; --waves) {
            const long long rest = blocks - waves * sms;
            for (int s = 2; rest > 0 && s <= 32; ++s) {
                const double t = waves * (pages + fixed) + (double)((rest * s + sms - 1) / sms) * (pages / s + fixed) + fixed;
                if (t < best) {
                    best = t;
                    full = waves * sms;
                    splits = s;
                }
            }
        }
        const size_t pieces = (size_t)(blocks - full) * splits;
        part_ml = align256(pieces * block * c->d * sizeof(float));
        total = part_ml + align256(pieces * block * sizeof(float2));
    }
};

// Rows per KV head from which the tensor-memory kernel is the faster one (us, decode kernel and it; 32 / 8 heads, d = 128, BF16): 8
// sequences of 4096, 8 rows 20.8 and 38.7, 16 31.0 and 39.4, 32 46.5 and 40.1, 128 133 and 46; 32 of 2048, 16 rows 52 and 66, 32 84
// and 68; one of 16384, 16 rows 23.8 and 26.2, 32 31.2 and 27.2; FP16, 16 of 1000, 16 rows 24.8 and 23.4; d = 64, FP16, 4 of
// 1500, 8 rows 10.4 and 13.6, 16 13.0 and 13.6.  d = 256, whose decode kernel takes 8 rows at a time: 8 of 4096, 8 rows 37 and 55, 16
// 57 and 56.  (One sequence of 300 takes 11 and 10 us at 2 to 8 rows; the host does not know lengths.)
bool tile_kernel_faster(int d, int rows) { return rows > (d == 256 ? 8 : 16); }

int run_tiles(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const CacheUnits& units, int rows,
              Strides qs, const void* q, const float* s, void* out, void* workspace, size_t workspace_bytes, int* d_status, void* stream,
              bool selftest = false)
{
    const TileLayout lay(cache, seqs->B, seqs->max_pages, rows);
    if (!workspace || workspace_bytes < lay.total || ((uintptr_t)workspace & 255)) return HIFA4_ERR_WORKSPACE;
    if (lay.blocks * 32 * lay.splits > 0x7FFFFFFFll) return HIFA4_ERR_UNSUPPORTED;
    const int rc = check_arch();
    if (rc) return rc;
    TileArgs a;
    std::memset(&a, 0, sizeof(a));
    common_args(a, cache, seqs, query, q, s, out, d_status);
    a.units = units;
    a.qs = qs;
    a.items = (int)lay.items;
    a.full = (int)lay.full;
    a.splits = lay.splits;
    a.part_o = (float*)workspace;
    a.part_ml = (float2*)((char*)workspace + lay.part_ml);
    const cudaError_t e = selftest ? launch_cache_attention_selftest(a, (cudaStream_t)stream)
                                   : launch_cache_attention(cache->in_dtype, cache->d, a, (cudaStream_t)stream);
    return e == cudaSuccess ? HIFA4_OK : HIFA4_ERR_CUDA;
}

// Workspace of a call; 0 where it is not built.
size_t attend_bytes(const hifa4_cache* cache, int B, int max_pages, const hifa4_cache_query* query, bool weight, bool many)
{
    CacheUnits units;
    int rows;
    if (!cache || cache->Hkv <= 0 || cache->Hkv > HIFA4_MAX_HEADS || !built(cache->d) || B <= 0 || max_pages <= 0) return 0;
    if (check_query(cache, query, &units, &rows)) return 0;
    if (many && tile_kernel_faster(cache->d, rows)) {
        const size_t n = TileLayout(cache, B, max_pages, rows).total;
        return n ? n : 256;
    }
    return DecodeLayout(cache, B, max_pages, query, rows, weight).total;
}

}  // namespace

extern "C" {

size_t hifa4_cache_page_bytes(int d) { return built(d) ? (size_t)74 * d : 0; }

int hifa4_cache_append(const hifa4_cache* cache, const hifa4_seqs* seqs, int n, const int* n_new, const void* k,
                       const hifa4_strides* k_strides, const void* v, const hifa4_strides* v_strides, const float* inv_s,
                       int* d_status, void* stream)
{
    count_call(1);
    int rc = check_cache(cache, true);
    if (rc) return rc;
    if ((rc = check_seqs(seqs, cache->Hkv))) return rc;
    if (n <= 0 || !factors_ok(inv_s)) return HIFA4_ERR_INVALID_ARG;
    Strides ks, vs;
    if ((rc = check_tensor(k, k_strides, cache->Hkv, n, cache->d, &ks))) return rc;
    if ((rc = check_tensor(v, v_strides, cache->Hkv, n, cache->d, &vs))) return rc;
    if ((rc = check_arch())) return rc;
    return launch_cache_append(cache->in_dtype, cache->d, view(cache, seqs, d_status), n, n_new, k, ks, v, vs, inv_s,
                               (cudaStream_t)stream) == cudaSuccess ? HIFA4_OK : HIFA4_ERR_CUDA;
}

int hifa4_cache_read(const hifa4_cache* cache, const hifa4_seqs* seqs, int n, const int* start, int out_dtype, void* k_out,
                     void* v_out, int* d_status, void* stream)
{
    int rc = check_cache(cache, false);
    if (rc) return rc;
    if ((rc = check_seqs(seqs, cache->Hkv))) return rc;
    if (n <= 0 || !k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15)) return HIFA4_ERR_INVALID_ARG;
    if (out_dtype < HIFA4_F16 || out_dtype > HIFA4_F32) return HIFA4_ERR_INVALID_ARG;
    if (out_dtype == HIFA4_F16) return HIFA4_ERR_UNSUPPORTED;        // does not hold every HIF4 value
    if ((rc = check_arch())) return rc;
    return launch_cache_read(cache->d, view(cache, seqs, d_status), n, start, out_dtype, k_out, v_out, (cudaStream_t)stream) ==
                   cudaSuccess ? HIFA4_OK : HIFA4_ERR_CUDA;
}

size_t hifa4_cache_decode_workspace_bytes(const hifa4_cache* cache, int B, int max_pages, const hifa4_cache_query* query,
                                          int with_page_weight)
{
    return query && query->N == 1 ? attend_bytes(cache, B, max_pages, query, with_page_weight != 0, false) : 0;
}

int hifa4_cache_decode(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
                       const hifa4_strides* q_strides, const float* s, void* out, float* lse, const float* page_weight,
                       float* page_weight_out, void* workspace, size_t workspace_bytes, int* d_status, void* stream)
{
    count_call(2);
    if (!query || query->N != 1 || (page_weight && !page_weight_out)) return HIFA4_ERR_INVALID_ARG;
    CacheUnits units;
    int rows;
    Strides qs;
    hifa4_strides one_token{};
    if (q_strides) one_token = hifa4_strides{q_strides->b, q_strides->h, 0};
    const int rc = check_call(cache, seqs, query, q, q_strides ? &one_token : nullptr, s, out, &units, &rows, &qs);
    if (rc) return rc;
    return run_decode(cache, seqs, query, units, rows, qs, q, s, out, lse, page_weight, page_weight_out, workspace, workspace_bytes,
                      d_status, stream);
}

size_t hifa4_cache_attention_workspace_bytes(const hifa4_cache* cache, int B, int max_pages, const hifa4_cache_query* query)
{
    return attend_bytes(cache, B, max_pages, query, false, true);
}

int hifa4_cache_attention(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
                          const hifa4_strides* q_strides, const float* s, void* out, void* workspace, size_t workspace_bytes,
                          int* d_status, void* stream)
{
    count_call(2);
    CacheUnits units;
    int rows;
    Strides qs;
    int rc = check_call(cache, seqs, query, q, q_strides, s, out, &units, &rows, &qs);
    if (rc) return rc;
    if (!tile_kernel_faster(cache->d, rows))
        return run_decode(cache, seqs, query, units, rows, qs, q, s, out, nullptr, nullptr, nullptr, workspace, workspace_bytes, d_status, stream);
    return run_tiles(cache, seqs, query, units, rows, qs, q, s, out, workspace, workspace_bytes, d_status, stream);
}

int hifa4_selftest_cache_wait_timeout(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
                                      void* out, float* page_weight_out, void* workspace, size_t workspace_bytes, int* d_status,
                                      void* stream)
{
    if (!d_status) return HIFA4_ERR_INVALID_ARG;
    CacheUnits units;
    int rows;
    Strides qs;
    const int rc = check_call(cache, seqs, query, q, nullptr, nullptr, out, &units, &rows, &qs);
    if (rc) return rc;
    if (cache->in_dtype != HIFA4_BF16 || cache->d != 128) return HIFA4_ERR_UNSUPPORTED;
    if (tile_kernel_faster(cache->d, rows)) {
        if (page_weight_out) return HIFA4_ERR_UNSUPPORTED;
        return run_tiles(cache, seqs, query, units, rows, qs, q, nullptr, out, workspace, workspace_bytes, d_status, stream, true);
    }
    if (decode_block_rows(cache->d, rows) != 8 || (page_weight_out && query->N != 1)) return HIFA4_ERR_UNSUPPORTED;
    return run_decode(cache, seqs, query, units, rows, qs, q, nullptr, out, nullptr, nullptr, page_weight_out, workspace, workspace_bytes,
                      d_status, stream, true);
}

int hifa4_cache_evict(const hifa4_seqs* seqs, const float* page_weight, int keep_pages, int keep_first, int keep_last,
                      int* block_table_out, int* kv_lens_out, float* page_weight_out, int* freed, int* n_freed,
                      int* d_status, void* stream)
{
    int rc = check_seqs(seqs, 1);
    if (rc) return rc;
    if (!page_weight || !block_table_out || !kv_lens_out || !page_weight_out || !freed || !n_freed) return HIFA4_ERR_INVALID_ARG;
    if (keep_first < 0 || keep_last < 1 || keep_pages < 0 || (long long)keep_first + keep_last > keep_pages) return HIFA4_ERR_INVALID_ARG;
    if ((rc = check_arch())) return rc;
    return launch_cache_evict(view(nullptr, seqs, d_status), page_weight, keep_pages, keep_first, keep_last, block_table_out,
                              kv_lens_out, page_weight_out, freed, n_freed, (cudaStream_t)stream) == cudaSuccess ? HIFA4_OK
                                                                                                                 : HIFA4_ERR_CUDA;
}

}  // extern "C"
