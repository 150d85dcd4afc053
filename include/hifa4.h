/*
 * hifa4.h -- C ABI of the HiFA4 hot path for NVIDIA B200 (sm_100a).
 *
 * HiFA4 (arxiv 2607.04302) runs both attention GEMMs, Q K^T and P V, on HIF4
 * 4-bit block-floating-point values, keeps the online-softmax state in FP16,
 * rescales post-RoPE Q and K per channel by calibration-static Smooth-QK
 * factors, and takes the softmax normalizer from the quantized P-hat that
 * feeds the PV GEMM (P-Reordering), produced in the same tensor-core pass by a
 * column of ones appended to V (Algorithm 1 "C4V16-Aux").
 *
 * Conventions for every entry point
 *   - All tensor pointers are DEVICE pointers owned by the caller unless a
 *     parameter says "host".  The library allocates no device memory, frees
 *     none and never synchronizes; work is enqueued on `stream`
 *     (a cudaStream_t passed as void*; NULL is the default stream).
 *   - Tensors are contiguous, row-major, in the index order given.
 *   - Return value: a hifa4_status.  No exception crosses this boundary and
 *     there is no CPU fallback: on a device that is not sm_100 every compute
 *     call returns HIFA4_ERR_ARCH.
 *   - `d_status` (optional, may be NULL) is a device int the kernels write a
 *     non-zero hifa4_status into when a bounded wait inside a kernel expires;
 *     the caller zeroes it and reads it after synchronizing.
 */
#ifndef HIFA4_H
#define HIFA4_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    HIFA4_OK = 0,
    HIFA4_ERR_INVALID_ARG = 1,   /* null pointer, non-positive size, bad enum          */
    HIFA4_ERR_UNSUPPORTED = 2,   /* shape / flag combination not built                 */
    HIFA4_ERR_WORKSPACE = 3,     /* workspace missing or too small                     */
    HIFA4_ERR_ARCH = 4,          /* current device is not compute capability 10.x      */
    HIFA4_ERR_CUDA = 5,          /* a CUDA runtime/driver call failed                  */
    HIFA4_ERR_TIMEOUT = 6        /* a bounded device-side wait expired (see d_status)  */
} hifa4_status;

typedef enum { HIFA4_F16 = 0, HIFA4_BF16 = 1, HIFA4_F32 = 2 } hifa4_dtype;

enum { HIFA4_Q = 0, HIFA4_K = 1, HIFA4_V = 2 };               /* `which` */
enum { HIFA4_PART_CODES = 0, HIFA4_PART_META = 1, HIFA4_PART_MMA = 2, HIFA4_PART_AUX = 3 }; /* `part` */
enum { HIFA4_MAX_HEADS = 256, HIFA4_MAX_DEBUG_BLOCKS = 16 };
enum { HIFA4_AGG_RMS = 0, HIFA4_AGG_MEAN = 0x100, HIFA4_AGG_P99 = 0x200 };   /* OR-ed into calibration `mode` */
#define HIFA4_STATIC_CALIB_MAX_FLOATS (1u << 20)   /* scratch limit of hifa4_smooth_calibrate_static */

/* Problem shape.  Q is [B,Hq,N,d]; K and V are [B,Hkv,N,d] ("GQA and batch
 * handling", Appendix "Implementation Details").  d in {64,128,256};
 * N a multiple of 64; Hq, Hkv <= HIFA4_MAX_HEADS.  q_to_kv is a HOST array of
 * Hq KV-head indices, or NULL for the usual grouping h / (Hq/Hkv) (then Hq
 * must be a multiple of Hkv).  in_dtype is HIFA4_F16 or HIFA4_BF16. */
typedef struct {
    int B, Hq, Hkv, N, d;
    const int* q_to_kv;
    int in_dtype;
} hifa4_shape;

/* Quantized Q/K/V (Algorithm 1 line 3).  Nine device buffers the caller
 * allocates with the sizes hifa4_quant_bytes() returns.
 *   *_codes : HIF4 element nibbles, two per byte, even element in the low
 *             nibble; nibble = sign<<3 | m, magnitude m/4 (S1P2).
 *   *_meta  : one uint32 per 64-element group: byte 0 the E6M2 level-1 scale
 *             code (S = 2^(e-48) (1+M/4), e = code>>2, M = code&3), byte 1
 *             the 8 level-2 bits (bit u covers elements 8u..8u+7), bytes 2-3
 *             the 16 level-3 bits (bit t covers elements 4t..4t+3).
 *             value_i = +-S * 2^(l2+l3) * m_i / 4      (Background, "HIF4").
 *   *_mma   : the same values, dequantized exactly to BF16 (every HIF4 value
 *             has at most 6 significant bits), in the layout the attention
 *             kernel's TMA loads expect.
 * Groups run along each GEMM's contraction axis: along d for Q and K
 * (codes [B,H,N,d/2], meta [B,H,N,d/64], mma [B,H,N,d]); along tokens for V
 * (codes [B,Hkv,d,N/2], meta [B,Hkv,d,N/64], mma [B,Hkv,d,N], i.e. V is
 * stored transposed).
 * Q-Mean auxiliary (Algorithm 1 lines 2 and 6; "Auxiliary Q-Mean Compensation"): when q_mu and
 * k_sum are both non-NULL, hifa4_quantize_qkv subtracts from every smoothed query token its mean
 * over the d channels before quantizing (the Q buffers then hold Q_z) and writes
 *   q_mu  [B,Hq,N]  floats: the per-token mean mu_i, an FP16 value;
 *   k_sum [B,Hkv,N] floats: sum over channels of the smoothed key, an FP16 value;
 * hifa4_attention_fwd with prm->qmean = 1 adds mu_i * k_sum_j to the raw score accumulators.
 * Leave both NULL for the path without Q-Mean.  (hifa4_quant_bytes: part HIFA4_PART_AUX.) */
typedef struct {
    uint8_t* q_codes; uint32_t* q_meta; void* q_mma;
    uint8_t* k_codes; uint32_t* k_meta; void* k_mma;
    uint8_t* v_codes; uint32_t* v_meta; void* v_mma;
    float* q_mu; float* k_sum;
} hifa4_qkv;

/* Calibration result summary (host memory).  rho_K and T_KQ are the gate
 * statistics of "Adaptive Applicability Gate"; this struct reports them as NaN
 * (hifa4_smooth_calibrate_auto computes them, into device memory).  branch: 0 bypass, 1 strong, 2 mild, 4 caller's alpha. */
typedef struct { float rho_K, T_KQ; int branch; float alpha; } hifa4_calib_stats;

/* Attention parameters.
 *   causal      1: key j contributes to row i only if j <= i.
 *   Br          query rows per CTA; scheduling only, must be 128.
 *   Bc          key-tile width of the online softmax (64 or 128).  It is part
 *               of the result: P is quantized under the running maximum that
 *               holds after each Bc keys (Algorithm 1 lines 7-10).
 *   normalizer  0: consistent (P-Reordering, normalizer = rowsum of P-hat via
 *               the ones column); 1: mismatched, the normalizer is accumulated
 *               from the unquantized FP16 P while PV consumes P-hat (the
 *               "Direct" baseline of "P-Reordering"; Theorem 1's O_mis).  Mode 1
 *               is an ablation: it runs on a one-thread-per-row kernel, several
 *               times slower than mode 0.
 *   qmean       1: add the Q-Mean correction mu_i * k_sum_j to the raw scores (line 6; scaled by the
 *               softmax scale together with them); needs qkv->q_mu and qkv->k_sum filled by
 *               hifa4_quantize_qkv.  0: no correction (the Q buffers must then hold un-centred Q).
 *   p_dtype     HIFA4_F16: exp(S-m) is rounded to FP16 before quantization
 *               ("FP16 operations", Appendix "Implementation Details").
 *               HIFA4_F32: variant that quantizes the FP32 exponential directly (a
 *               different function: it changes a few 1e-4 of the P-hat codes); built
 *               for Bc = 64 with d = 128 or 256 and the consistent normalizer,
 *               HIFA4_ERR_UNSUPPORTED elsewhere.
 *   out_dtype   HIFA4_F16 / HIFA4_BF16 / HIFA4_F32 element type of `out`.
 *   softmax_scale  0 selects 1/sqrt(d). */
typedef struct {
    int causal, Br, Bc;
    int normalizer, qmean, p_dtype, out_dtype;
    float softmax_scale;
} hifa4_attn_params;

/* Optional debug dump of P-hat for up to HIFA4_MAX_DEBUG_BLOCKS 128-row query
 * blocks.  blocks: HOST array of n_blocks triples (b, h, query_block_index).
 * p_codes: device [n_blocks][128][N] bytes, the nibble of every P-hat element
 * (0 where the key tile was skipped by causality); p_step: device
 * [n_blocks][128][N/4] floats, the step of every 4-key subgroup (0 for an all-zero group); l_out, m_out:
 * device [n_blocks][128] floats, the accumulated normalizer and the final
 * running maximum.  Any of the four device pointers may be NULL. */
typedef struct {
    int n_blocks;
    const int* blocks;
    uint8_t* p_codes;
    float* p_step;
    float* l_out;
    float* m_out;
} hifa4_debug;

/* Histogram of the per-tile mass error of P-hat ("P-Reordering", Theorem 1 and the
 * figure of its empirical validation): for every query row and every Bc-key tile whose
 * P is not all zero, eps = sum_j P-hat_j / sum_j P_j - 1 over the keys of the tile, both
 * sums exact.  hist: device array of n_bins + 2 counters that the call ADDS to (clear it
 * first): bin k counts lo + k*w <= eps < lo + (k+1)*w with w = (hi - lo)/n_bins; entry
 * n_bins counts eps < lo, entry n_bins + 1 counts eps >= hi. */
typedef struct {
    unsigned long long* hist;
    int n_bins;
    double lo, hi;
} hifa4_mass_stats;

const char* hifa4_status_string(int status);

/* Self-test of the failure path of the device-side waits (no counterpart in the paper; for deployment
 * checks and for the test-suite).  Launches the Bc = 64, d = 128 attention kernel that a call with these
 * arguments would take (the one with two query blocks per CTA for large problems) in an instantiation
 * whose softmax warps withhold the arrival that releases the P V product and whose issuer gives up
 * waiting for it after 2^6 polls (at most a fraction of a millisecond) instead of 2^18.  That wait begins
 * only when every TMA load has landed and no MMA is in flight.  When it runs out the kernel records
 * HIFA4_ERR_TIMEOUT + 16 * 7 (site 7: the issuer's wait for P V) in *d_status (required, device int, zero on
 * entry), raises the CTA's abort flag, every role leaves through the common exit that frees tensor memory, and
 * the call returns normally.
 * `out` is not written.  Arguments as hifa4_attention_fwd (prm: Bc = 64, no variant flags; shape: d = 128);
 * the test-suite uses a one-CTA problem (N <= 128, one head) and some with hundreds of CTAs.  Nothing hangs, faults or traps. */
int hifa4_selftest_wait_timeout(const hifa4_shape* shape, const hifa4_qkv* qkv, const hifa4_attn_params* prm,
                                void* out, int* d_status, void* stream);

/* Calls made so far in this process: out[0] calibrate, out[1] quantize (hifa4_cache_append too),
 * out[2] attention (hifa4_cache_decode and hifa4_cache_attention too), out[3] kernels launched (all entry points). */
void hifa4_get_counters(unsigned long long out[4]);

/* Offline Smooth-QK calibration (Eq. "sqk"; "Calibration-Static Deployment").
 *   q_cal [S,Hq,Ncal,d], k_cal [S,Hkv,Ncal,d]: post-RoPE calibration
 *   activations of one layer, S samples of Ncal tokens, element type dt.
 *   Per sample and channel the statistic is the largest magnitude over tokens
 *   (for Q also over the query heads sharing the KV head); samples are
 *   combined by root-mean-square; s = Kagg^alpha / Qagg^(1-alpha), 1 where an
 *   aggregate is zero.  mode: 0 bypass (s = 1), 1 strong (alpha 0.5), 2 mild
 *   (alpha 0.25), 4 caller's alpha; 3 (gate decides) returns
 *   HIFA4_ERR_UNSUPPORTED here: use hifa4_smooth_calibrate_auto, which takes
 *   the extra scratch the gate statistics need.  OR-ing HIFA4_AGG_MEAN or
 *   HIFA4_AGG_P99 into mode replaces the root-mean-square over samples by the
 *   mean or by the nearest-rank 99th percentile of the per-sample maxima (the
 *   two alternatives of the paper's aggregator comparison, table "calib").
 *   Outputs (device): s, inv_s [Hkv,d] floats, inv_s = fl32(1/s).
 *   absmax_ws: device scratch of 2*S*Hkv*d floats; the call clears it.
 *   host_stats: optional HOST struct, filled without synchronizing. */
int hifa4_smooth_calibrate(const void* q_cal, const void* k_cal, int S, int Hq, int Hkv,
                           int Ncal, int d, const int* q_to_kv, int dt, int mode, float alpha,
                           float* s, float* inv_s, float* absmax_ws,
                           hifa4_calib_stats* host_stats, void* stream);

/* Calibration with the applicability gate deciding the branch ("Adaptive Applicability
 * Gate"), entirely on the device:
 *   rho_K = max|K| / P99(|K|), the 99th percentile (nearest rank) over every element of
 *   k_cal, read off an exact histogram of the 15-bit magnitude patterns;
 *   T = max|K| / max|Q| over every element of k_cal and q_cal;
 *   rho_K >= 6 and T >= 2 select Smooth-QK, with alpha = 0.5 (strong) if T > 3 and
 *   alpha = 0.25 (mild) if 2 <= T <= 3; anything else bypasses (s = 1).
 * Arguments as hifa4_smooth_calibrate, plus
 *   gate_ws : device scratch of HIFA4_GATE_WS_BYTES bytes, 8-byte aligned;
 *   d_stats : NULL, or DEVICE array of 4 floats that receives rho_K, T, the branch
 *             (0 bypass, 1 strong, 2 mild) and alpha.  The call does not synchronize: copy
 *             the four floats back after the stream has run if the host wants them.
 * S*Hkv*Ncal*d must be below 2^32 (HIFA4_ERR_UNSUPPORTED otherwise). */
#define HIFA4_GATE_WS_BYTES (32768u * 4u + 64u)
int hifa4_smooth_calibrate_auto(const void* q_cal, const void* k_cal, int S, int Hq, int Hkv,
                                int Ncal, int d, const int* q_to_kv, int dt, float* s,
                                float* inv_s, float* absmax_ws, void* gate_ws, float* d_stats,
                                void* stream);

/* hifa4_smooth_calibrate for callers that cannot allocate device memory.
 * (The paper has no counterpart: this entry point exists for deployment only.)
 *   Who needs it: code that runs where cudaMalloc is off limits -- a serving process whose whole
 *   device memory already belongs to an arena it may not grow, a plug-in called from a runtime
 *   that forbids allocation on its worker threads, a latency-critical section that cannot take
 *   the device-wide synchronization an allocation implies.  Such a caller still owns its inputs
 *   and outputs (q_cal, k_cal, s, inv_s) but has nowhere to get the 2*S*Hkv*d-float scratch from.
 *   What it does: the same computation, with the same kernels, as hifa4_smooth_calibrate; the
 *   scratch is a fixed array of HIFA4_STATIC_CALIB_MAX_FLOATS floats (4 MiB) in device global
 *   memory, which every GPU that loads this library holds until the process exits.  The call
 *   makes no cudaMalloc/cudaFree and uses no allocating library routine.
 *   Limits and rules:
 *   - 2*S*Hkv*d must not exceed HIFA4_STATIC_CALIB_MAX_FLOATS, else HIFA4_ERR_WORKSPACE is
 *     returned and nothing is enqueued (use hifa4_smooth_calibrate with your own workspace).
 *   - The first call on each device looks up the device address of the array (with that device
 *     current).  Make that first call outside any stream capture.
 *   - All calls on a device share the one array, which keeps the previous call's contents; each
 *     call clears the part it uses before reducing into it.  Two calls whose kernels may overlap
 *     on the GPU (different streams, no ordering between them) race on it: serialize them.
 *   Arguments and results otherwise as hifa4_smooth_calibrate, minus absmax_ws. */
int hifa4_smooth_calibrate_static(const void* q_cal, const void* k_cal, int S, int Hq, int Hkv,
                                  int Ncal, int d, const int* q_to_kv, int dt, int mode,
                                  float alpha, float* s, float* inv_s,
                                  hifa4_calib_stats* host_stats, void* stream);

/* Bytes of one buffer of hifa4_qkv for this shape; 0 on a bad argument. */
size_t hifa4_quant_bytes(const hifa4_shape* shape, int which, int part);

/* Smooth-QK scaling fused with HIF4 quantization (Algorithm 1 lines 1 and 3).
 *   q~ = round_in(q * s[kv(h)]), k~ = round_in(k * inv_s[g]) with an fp32
 *   multiply rounded to the input dtype; V is quantized as it is.
 *   s, inv_s: [Hkv,d] floats, or both NULL for bypass.  Any of q, k, v may be
 *   NULL to skip that tensor.  Fills the buffers of `out`. */
int hifa4_quantize_qkv(const hifa4_shape* shape, const void* q, const void* k, const void* v,
                       const float* s, const float* inv_s, const hifa4_qkv* out,
                       int* d_status, void* stream);

/* Workspace the attention call needs (may be 0). */
size_t hifa4_attention_workspace_bytes(const hifa4_shape* shape, const hifa4_attn_params* prm);

/* Fused prefill attention forward on quantized operands (Algorithm 1 lines
 * 4-13): S = Q-hat K-hat^T / sqrt(d); FP16 running max and rescale;
 * P = exp(S - m) in FP16; P-hat = HIF4(P) per row and 64 keys;
 * [O | l] += P-hat [V-hat | 1]; out = O / l.
 *   qkv: buffers filled by hifa4_quantize_qkv for the same shape (only the
 *   *_mma images are read).  out: [B,Hq,N,d] of prm->out_dtype.
 *   workspace: at least hifa4_attention_workspace_bytes() bytes (NULL if 0).
 *   dbg: NULL, or a P-hat dump request.
 * Scheduling note (calibration and quantization alike): the grids are launched
 * with programmatic stream serialization (all but those of the 128-key and the
 * one-thread-per-row kernel), i.e. their CTAs may become resident while the
 * preceding kernel of the stream is still draining; the status word aside, they
 * read and write no global memory before that kernel has completed, so the usual
 * stream order of results holds. */
int hifa4_attention_fwd(const hifa4_shape* shape, const hifa4_qkv* qkv,
                        const hifa4_attn_params* prm, void* out, void* workspace,
                        const hifa4_debug* dbg, int* d_status, void* stream);

/* hifa4_attention_fwd that also fills the mass-error histogram of P-hat (see
 * hifa4_mass_stats; "P-Reordering", Theorem 1).  Same arguments and result as
 * hifa4_attention_fwd (either normalizer mode); stats must be non-NULL with
 * n_bins >= 1 and lo < hi.  Analysis path: it runs on the one-thread-per-row kernel. */
int hifa4_attention_fwd_stats(const hifa4_shape* shape, const hifa4_qkv* qkv,
                              const hifa4_attn_params* prm, void* out, void* workspace,
                              const hifa4_mass_stats* stats, int* d_status, void* stream);

/* hifa4_attention_fwd with Algorithm 1 line 1 inside the attention kernel: q is
 * the raw post-RoPE Q [B,Hq,N,d] of shape->in_dtype (device), s the Smooth-QK
 * factors of Q [Hkv,d] (device) or NULL; every CTA smooths and HIF4-quantizes
 * its own 128 query rows in shared memory, so Q-hat is never written to device
 * memory (its codes are not produced).  kv: buffers filled by
 * hifa4_quantize_qkv(shape, NULL, k, v, ...) for the same shape (only k_mma
 * and v_mma are read).  The result is bit-identical to hifa4_quantize_qkv on
 * q followed by hifa4_attention_fwd.  Supported for Bc = 64, d = 128,
 * qmean = 0, normalizer = 0; anything else returns HIFA4_ERR_UNSUPPORTED
 * without a launch.  Other arguments, status word and scheduling note as
 * hifa4_attention_fwd. */
int hifa4_attention_fwd_qraw(const hifa4_shape* shape, const void* q, const float* s,
                             const hifa4_qkv* kv, const hifa4_attn_params* prm, void* out,
                             void* workspace, int* d_status, void* stream);

/* Experiment, not a default path: hifa4_attention_fwd with S = Q-hat K-hat^T issued
 * as tcgen05.mma kind::f8f6f4 (the 8-bit MMA kind nearest to the "HIF4 Cube" of
 * Algorithm 1's comments).  Element x micro-exponent (an integer up to 28) is exact
 * in E4M3; the E6M2 group scale is not, so S is accumulated separately per
 * 64-channel group and the two partial sums are combined with the FP32 group
 * scales by the softmax threads (exact products, one rounding).  The call first
 * derives the E4M3 images and group scales of Q and K from qkv's packed codes and
 * metadata into `workspace` (hifa4_f8qk_workspace_bytes(), 256-byte aligned), then
 * runs the attention kernel; P V is unchanged (v_mma is read).  d = 128, Bc = 64,
 * qmean = 0, normalizer = 0, p_dtype = F16; anything else returns
 * HIFA4_ERR_UNSUPPORTED.  The result meets the same bars against the oracle as
 * hifa4_attention_fwd (the scores are the correctly rounded exact sums). */
size_t hifa4_f8qk_workspace_bytes(const hifa4_shape* shape);
int hifa4_attention_fwd_f8qk(const hifa4_shape* shape, const hifa4_qkv* qkv,
                             const hifa4_attn_params* prm, void* out, void* workspace,
                             size_t workspace_bytes, int* d_status, void* stream);

/* Workspace for hifa4_attention_fwd_raw: all hifa4_qkv buffers (each rounded up
 * to 256 bytes; the two Q-Mean vectors only when prm->qmean = 1) plus the
 * attention workspace. */
size_t hifa4_attention_raw_workspace_bytes(const hifa4_shape* shape, const hifa4_attn_params* prm);

/* Algorithm 1 end to end on raw post-RoPE Q/K/V: hifa4_quantize_qkv into
 * `workspace`, then hifa4_attention_fwd (same result).  What the workspace holds
 * afterwards is not defined: only the operand images that the attention kernel
 * reads are formed, no codes and no metadata, and for large problems that
 * hifa4_attention_fwd_qraw supports those of K and V only, Q being quantized
 * inside the attention kernel.  s, inv_s as in hifa4_quantize_qkv. */
int hifa4_attention_fwd_raw(const hifa4_shape* shape, const void* q, const void* k, const void* v,
                            const float* s, const float* inv_s, const hifa4_attn_params* prm,
                            void* out, void* workspace, size_t workspace_bytes,
                            int* d_status, void* stream);

/* ---------------------------------------------------------------------------
 * Serving: a paged HIF4 key-value cache, and attention over it.
 *
 * A page holds HIFA4_PAGE_TOKENS = 64 consecutive tokens of one sequence, for every KV head: one HIF4 group of V per
 * channel.  The pool is one buffer of n_pages * Hkv * hifa4_cache_page_bytes(d) bytes, [n_pages][Hkv][74 d] (16-byte
 * aligned): per value 4 bits of code, 0.5 bits of micro-exponents and 0.125 bits of scale.  Per page and head, in bytes:
 *   K codes  32 d  [64][4][d/64][2] words: units 2p and 2p+1 (8 elements each) of group G of a token at [token][p][G];
 *                  element e of the unit in nibble e, nibble = 8 + signed code (value = code * S/4 * 2^shift)
 *   K shifts  4 d  [64][d/64] words: the shift (0..2) of the 4-element subgroup 2u+r in bits 16r+2u and 16r+2u+1
 *   K scales    d  [64][d/64] bytes: E6M2 code of S
 *   V codes  32 d  [d][8] words: word 2i+h has the tokens 16i+4h+(0..3) in nibbles 0..3, 16i+8+4h+(0..3) in nibbles 4..7
 *   V shifts  4 d  [d] words: the shift of nibbles 4r..4r+3 of word w in bits 16r+2w and 16r+2w+1
 *   V scales    d  [d] bytes
 * Scales, shifts and codes are those of hifa4_quantize_qkv (a NaN is stored as zero); tokens behind the end of a sequence
 * count as zeros in V's groups.  Both halves of the metadata that a lane needs for 8 codes are two bits wide, which is why
 * the shifts take 32 instead of 24 bits per group.
 * V's groups run along tokens, so the group of an incomplete page changes with every token.  v_tail keeps the raw values of
 * the tokens in a sequence's incomplete page, row = position in the page: [n_tails][Hkv][64][d] elements of in_dtype.  It is
 * read and written by hifa4_cache_append only and may be NULL for the other calls.
 *
 * hifa4_seqs: B sequences.  block_table [B][max_pages]: physical page of each logical page; kv_lens [B]: tokens of each
 * sequence (0 allowed), for hifa4_cache_append including the new ones; tail_slots [B]: a sequence's row of v_tail, NULL: its
 * index.  All three are DEVICE arrays, so that captured graphs can be replayed with other contents; a length, page or slot
 * out of range is found on the device: its sequence (a page: its tokens) is left out, and *d_status is set to
 * HIFA4_ERR_INVALID_ARG, unless it holds a code already (that of an expired wait is never lost).  Block tables of different
 * sequences may share pages for reading; no two sequences of one hifa4_cache_append may write the same page or tail.
 *
 * hifa4_strides: distance in elements between consecutive batch rows, heads and tokens of a 16-bit tensor whose channels are
 * contiguous; multiples of 8, the tensor 16-byte aligned.  NULL: contiguous [B][H][tokens][d].  Factors (s, inv_s) and the
 * outputs of hifa4_cache_read are 16-byte aligned.  Outputs and workspaces overlap no input and not one another, except where a call
 * says that they may be the same array.
 *
 * Sizes: B * Hkv up to 65535, max_pages up to 2^24, N up to 2^20, (2 max_pages + 1) * B * Hkv * (blocks of 8 or 16 query rows per KV head)
 * up to 2 * 10^9 for attention of few query rows; beyond them HIFA4_ERR_UNSUPPORTED.  Kernels read a table only as far as its sequences reach,
 * but its width is all that the host knows of their lengths: it sets the workspaces (page weights: 8 B Hq max_pages bytes) and how
 * hifa4_cache_attention shares its work out.
 * ------------------------------------------------------------------------- */
enum { HIFA4_PAGE_TOKENS = 64 };
typedef struct {
    int Hkv, d, in_dtype;
    int n_pages;
    void* pages;
    int n_tails;
    void* v_tail;
} hifa4_cache;
typedef struct {
    int B, max_pages;
    const int* block_table;
    const int* kv_lens;
    const int* tail_slots;
} hifa4_seqs;
typedef struct { long long b, h, t; } hifa4_strides;

/* Bytes of one KV head's part of a page, 74 d; 0 for a d that is not built (64, 128, 256 are). */
size_t hifa4_cache_page_bytes(int d);

/* Smooth-QK and HIF4 quantization of new tokens into the cache: k, v [B,Hkv,n,d] of cache->in_dtype; sequence b takes its
 * first n_new[b] tokens (device array; NULL: n of them; 0 allowed) at positions kv_lens[b] - n_new[b] and on.  inv_s: [Hkv,d]
 * factors of K as in hifa4_quantize_qkv, or NULL.
 * The older values of a page that is continued come from v_tail.  An append leaves there what the last page may be continued from: the
 * rows of an incomplete page, and of a page that it completes but did not begin all but the last.  So before the next append a
 * sequence may be cut back (kv_lens lowered: drafted tokens that were not accepted)
 *   - to any multiple of 64: the tokens behind it are appended anew;
 *   - inside its last page, unless that is full and one append filled it from its first position on.
 * Further back, inside another page, it may not: V's groups would be formed again from rows that v_tail does not hold.  A draft that
 * crosses into the next page is settled by cutting the sequence back to the first position of the page that it left and appending
 * that page's accepted tokens again, whose K and V the caller has to have. */
int hifa4_cache_append(const hifa4_cache* cache, const hifa4_seqs* seqs, int n, const int* n_new, const void* k,
                       const hifa4_strides* k_strides, const void* v, const hifa4_strides* v_strides, const float* inv_s,
                       int* d_status, void* stream);

/* The values that the cache holds: token i of row b of k_out, v_out [B,Hkv,n,d] (HIFA4_BF16 or HIFA4_F32: both hold every HIF4
 * value exactly) is the one at position start[b] + i (device array; NULL: 0).  Rows at or behind kv_lens[b] are left as they were. */
int hifa4_cache_read(const hifa4_cache* cache, const hifa4_seqs* seqs, int n, const int* start, int out_dtype, void* k_out,
                     void* v_out, int* d_status, void* stream);

/* What the attention calls ask: Hq query heads (q_to_kv as in hifa4_shape: HOST array or NULL), N query tokens per sequence,
 * causal (hifa4_cache_attention only): query i of a sequence of length L sees the keys up to position L - N + i; otherwise all L.
 * A query that sees no key gets zeros.  softmax_scale 0 selects 1/sqrt(d).  `out` of the calls is 16-byte aligned. */
typedef struct {
    int Hq;
    const int* q_to_kv;
    int N, causal, out_dtype;
    float softmax_scale;
} hifa4_cache_query;

/* Attention of one new token per sequence over the cache: out [B,Hq,d] = softmax(q~ K^T scale) V on the cache's values, with
 * q~ = round_in(q * s) (q [B,Hq,d] of cache->in_dtype, q_strides->t unused; s [Hkv,d] or NULL) not quantized: q is a
 * vanishing part of what a step reads.  Softmax in FP32; P enters the product with V in FP16, scaled to 2^15 at the running maximum.
 *   lse             [B,Hq] floats or NULL: log(sum_j exp(score_j)), -inf without keys
 *   page_weight_out [B][max_pages] floats or NULL: page_weight (NULL: zeros; may be the same array) plus the attention weight that
 *                   the page's tokens got, summed over the query heads.  Entries behind a sequence's last page are left as they were.
 * query->N must be 1.  workspace: hifa4_cache_decode_workspace_bytes() bytes, 256-byte aligned, its contents irrelevant
 * before and after; calls that may overlap need one each.  Sums are taken in a fixed order: equal calls give equal bits. */
size_t hifa4_cache_decode_workspace_bytes(const hifa4_cache* cache, int B, int max_pages, const hifa4_cache_query* query,
                                          int with_page_weight);
int hifa4_cache_decode(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
                       const hifa4_strides* q_strides, const float* s, void* out, float* lse, const float* page_weight,
                       float* page_weight_out, void* workspace, size_t workspace_bytes, int* d_status, void* stream);

/* The same for N >= 1 query tokens per sequence: q [B,Hq,N,d], out [B,Hq,N,d].  Cross attention to an encoder's states of other
 * lengths (causal 0), the next chunk of a prompt or several drafted tokens (causal 1, after their append; hifa4_cache_append says how far
 * they can be taken back).  More than 16 query rows (heads times tokens; d = 256: 8) per KV head take a kernel on tcgen05 in which P is
 * rounded to BF16, for FP16 activations to two terms of BF16 (16 bits).  The workspace may be used by the next call on the same stream. */
size_t hifa4_cache_attention_workspace_bytes(const hifa4_cache* cache, int B, int max_pages, const hifa4_cache_query* query);
int hifa4_cache_attention(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
                          const hifa4_strides* q_strides, const float* s, void* out, void* workspace, size_t workspace_bytes,
                          int* d_status, void* stream);

/* Self-test of the failure path of the two calls' device waits, as hifa4_selftest_wait_timeout: the kernel that hifa4_cache_attention
 * would take (with page_weight_out: hifa4_cache_decode), in an instantiation whose first CTA's loader leaves a page out (the second
 * page of its first consumer warp; the third page of a CTA of the kernel on tcgen05) and whose wait for that page ends after 2^6 polls.
 * *d_status (required, zero on entry) becomes HIFA4_ERR_TIMEOUT; what depends on that CTA is not written or undefined, all else is as
 * in the ordinary call.  Built for BF16, d = 128 and, of the decode kernel, up to 8 query rows per KV head; q is contiguous. */
int hifa4_selftest_cache_wait_timeout(const hifa4_cache* cache, const hifa4_seqs* seqs, const hifa4_cache_query* query, const void* q,
                                      void* out, float* page_weight_out, void* workspace, size_t workspace_bytes, int* d_status,
                                      void* stream);

/* Eviction by accumulated attention weight, whole pages (single tokens would break V's groups).  A sequence of more than
 * keep_pages pages keeps its first keep_first, its last keep_last (>= 1: the incomplete page stays) and, of those between, the
 * keep_pages - keep_first - keep_last with the largest page_weight (equal weights: the lower index; a NaN counts as less than
 * everything).  Kept pages close ranks in their order; positions inside K are those of its rotary embedding and stay.
 *   block_table_out, page_weight_out [B][max_pages], kv_lens_out [B]: may be the inputs themselves; entries behind the last
 *                   page become -1 and 0;
 *   freed [B][max_pages], n_freed [B]: physical pages that left the table, in order, -1 behind the last.
 * seqs->tail_slots is not used.  A sequence whose length is out of range keeps all (see above). */
int hifa4_cache_evict(const hifa4_seqs* seqs, const float* page_weight, int keep_pages, int keep_first, int keep_last,
                      int* block_table_out, int* kv_lens_out, float* page_weight_out, int* freed, int* n_freed,
                      int* d_status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HIFA4_H */
