/*
 * grinqh.h -- C ABI of libgrinqh, the nested-precision decode VMM of GRINQH
 * (Graded Input-based Quantization Hierarchy, arXiv 2606.23419) for AMD
 * Instinct MI355X (gfx950).
 *
 * The path (Sec. 3 of the paper):
 *   offline   W (fp16) --RTN, 8 bits, group 128--> codes + scales
 *             codes --nest + pack--> bit planes, most significant first
 *   per token x --magnitude grading--> a level per input channel
 *             y = W_hat(levels) x, each weight row read only to the depth its
 *             channel's level asks for (Sec. 3.3 "Storage Layout and Weight
 *             Loading"; App. C.1 "Sparse bit-loading").
 *
 * Conventions for every entry point
 *   - Device pointers are plain HIP device addresses owned by the caller; the
 *     library never allocates, frees or synchronises.  Host pointers are read
 *     during the call only.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     All work is enqueued on it; nothing waits for it.
 *   - Every argument is validated on the host before anything is enqueued; a
 *     failing call returns a negative status, writes nothing and leaves a
 *     message for grinqh_last_error().  A failing launch returns GRINQH_EHIP.
 *     Faults inside kernels surface at the caller's next synchronisation.
 *   - Calls are thread-safe; the error message is per thread.
 *
 * Packed layout (the contract between grinqh_pack and grinqh_vmm)
 *   b_max (the top level's bits) in {4, 6, 8}: codes q are b_max-bit offset
 *   binary, w_hat = s*(q - 2^(b_max-1)) at full depth (Sec. 3.3 stores b_max
 *   = 4, 6 or 8).  u (plane_bits) in {1, 2}; P = b_max/u planes; T (tile_n)
 *   outputs per tile; R = T*b_max/8 bytes per stored row.
 *   codes buffer: (N/T) tiles x K rows x R bytes = K*N*b_max/8 bytes.
 *   Row (tile t, channel k) starts at byte (t*K + k)*R.  Plane j (1-based,
 *   j = 1 most significant) starts at byte (j-1)*T*u/8 of the row and holds,
 *   for local output o = n - t*T, the field (q >> (b_max - j*u)) & (2^u - 1)
 *   at bit o*u of the plane (byte floor(o*u/8), bit (o*u) % 8, little-endian).
 *   Reading b bits of a channel therefore reads the first b*T/8 bytes of its
 *   row in every tile: a contiguous prefix, a multiple of 64 bytes.
 *   scales buffer: fp16 [K/128][N], the scale of group g for output n at
 *   index g*N + n.
 */
#ifndef GRINQH_H
#define GRINQH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define GRINQH_API __attribute__((visibility("default")))
#else
#define GRINQH_API
#endif

typedef enum {
  GRINQH_OK = 0,
  GRINQH_EINVAL = -1,       /* invalid argument: null pointer, bad shape, bad ordering */
  GRINQH_EUNSUPPORTED = -2, /* well-formed but outside what these kernels implement */
  GRINQH_ESIZE = -3,        /* workspace too small, or a size overflows */
  GRINQH_EHIP = -4          /* the HIP runtime reported an error at launch */
} grinqh_status;

#define GRINQH_MAX_LEVELS 9

/* Layer descriptor: 36 bytes, natural alignment, no implicit padding. */
typedef struct {
  int32_t K;          /* input channels (d_in); a multiple of `group` */
  int32_t N;          /* outputs (d_out); a multiple of the tile width */
  int32_t group;      /* quantisation group along K; must be 128 */
  int32_t n_levels;   /* number of levels n+1 including level 0; 2..9 */
  uint8_t level_bits[GRINQH_MAX_LEVELS];
                      /* b_0 = 0 < b_1 < ... < b_n = b_max (Sec. 3.1: the set
                         B); b_max in {4, 6, 8} is the stored code width;
                         every b_i a multiple of plane_bits */
  uint8_t reserved_[3];
  int32_t plane_bits; /* u: 0 = auto (2 if every b_i is even, else 1); or 1, 2 */
  int32_t tile_n;     /* T: 0 = auto; else 256, 512, 1024 or 2048 with T*u >= 512 */
} grinqh_layer_desc;

enum { GRINQH_SRC_FP16_RTN = 0, GRINQH_SRC_CODES_U8 = 1 };
enum { GRINQH_ASSIGN_THRESHOLD = 0, GRINQH_ASSIGN_TOPK = 1 };
enum { GRINQH_VMM_ACCUMULATE = 1 };
/* Options of grinqh_set_option, and the kernels GRINQH_OPT_VMM_KERNEL names. */
enum { GRINQH_OPT_VMM_KERNEL = 1, GRINQH_OPT_GROUPS_PER_WG = 2, GRINQH_OPT_PREFILL_TILE = 3,
       GRINQH_OPT_LUT_GROUPS = 4, GRINQH_OPT_PREFILL_CUS = 5, GRINQH_OPT_ATTEND_KERNEL = 6,
       GRINQH_OPT_ATTEND_SPLITS = 7 };
enum { GRINQH_ATTEND_ROWS = 1, GRINQH_ATTEND_TILE = 2 };
enum { GRINQH_KERNEL_AUTO = 0, GRINQH_KERNEL_PER_PLANE = 1, GRINQH_KERNEL_GENERAL = 2 };

/* Infrastructure, not an operation of the paper.  Fill the auto fields
 * (plane_bits, tile_n) of *in into *out after validating it.  Host only.
 * Every other entry point resolves the same way. */
GRINQH_API int grinqh_resolve_desc(const grinqh_layer_desc* in, grinqh_layer_desc* out);

/* Infrastructure, not an operation of the paper: sizes of the packed buffers
 * of a layer (host only), codes K*N*b_max/8 bytes, scales 2*(K/128)*N bytes. */
GRINQH_API int grinqh_packed_bytes(const grinqh_layer_desc* desc, size_t* codes_bytes,
                        size_t* scales_bytes);

/* Offline quantise + nest + pack (Sec. 3.3, App. C.1).
 *   src_kind GRINQH_SRC_FP16_RTN: src = fp16 W[N][K] (torch Linear.weight
 *     layout), src_scales = NULL.  Symmetric RTN at b_max bits per (output,
 *     group of 128 channels), with h = 2^(b_max-1): s = fp16_rne(fp32(max|w|)
 *     / (h - 1)), q = clamp(rne(w/s), -h, h - 1) + h; a group with s == 0
 *     gets q = h.  W must be finite.
 *   src_kind GRINQH_SRC_CODES_U8: src = uint8 codes q[N][K] (q < 2^b_max;
 *     higher bits are ignored) from any base quantiser with the same
 *     offset-binary convention, src_scales = fp16 s[N][K/128] (the method is
 *     quantisation-agnostic, Sec. 3.3).  Codes of the look-up-table format
 *     (grinqh_vmm_lut) have no scales: pass src_scales = packed_scales = NULL.
 *   Outputs: packed_codes (K*N*b_max/8 bytes, layout above), packed_scales
 *   (fp16 [K/128][N]).  Inputs and outputs must not overlap. */
GRINQH_API int grinqh_pack(const grinqh_layer_desc* desc, int src_kind, const void* src,
                const void* src_scales, void* packed_codes, void* packed_scales,
                void* stream);

/* Integer channel counts for a precision distribution P given in basis
 * points (p_0..p_n, each >= 0, summing to 10000; App. A.1).  With
 * U_j = sum_{i>=j} p_i, C_j = floor((U_j*K + 5000)/10000) channels get level
 * >= j; counts_out[j] = C_j - C_{j+1} (n+1 values summing to K).  Host only. */
GRINQH_API int grinqh_topk_counts(int32_t K, int32_t n_levels, const int32_t* p_bp,
                       int32_t* counts_out);
/* (p_bp and counts_out each hold exactly n_levels entries.) */

/* Infrastructure, not an operation of the paper: device workspace needed by
 * grinqh_assign / grinqh_vmm for B tokens.  The present kernels need none and
 * report 0; callers may pass NULL/0. */
GRINQH_API int grinqh_workspace_bytes(const grinqh_layer_desc* desc, int32_t B, size_t* bytes);

/* Offline threshold calibration (Sec. 3.2 calibration of the thresholds;
 * App. A.1).  x: fp16 [S][K] (device) calibration activations, one sample per
 * row, finite; p_bp: host int32 p_0..p_n in basis points (each >= 0, summing
 * to 10000; exactly n_levels entries are read).  For each sample and each
 * k = 1..n (n = n_levels-1) the sample threshold is the type-7 sample
 * quantile of |x| at q_k = U_k / 10000, U_k = p_0 + .. + p_(k-1): with the K
 * magnitudes sorted ascending a_0 <= .. <= a_(K-1), h = (K-1) U_k / 10000 is
 * split exactly into lo = floor(h) and frac = (h - lo) as a float64 quotient
 * of integers, and the threshold is a_lo + frac * (a_(lo+1) - a_lo) in
 * float64 (a_(lo+1) = a_lo at lo = K-1).  theta_k is the float64 mean of the
 * sample thresholds, summed in sample order, rounded to fp32.
 *   per_sample: device float64 [S][n] scratch, written (8-byte aligned).
 *   theta: device fp32 [n] out.  Requires 1 <= S <= 65535, K <= 16384. */
GRINQH_API int grinqh_calibrate(const grinqh_layer_desc* desc, const void* x, int32_t S,
                                const int32_t* p_bp, double* per_sample, float* theta,
                                void* stream);

/* grinqh_calibrate for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the per-sample scratch lives in a static device array of the library
 * (1 MiB, float64, each GPU holds its own until the process ends), so the
 * caller passes no workspace.  Arguments and result as grinqh_calibrate;
 * S * (n_levels - 1) must not exceed 131072 (GRINQH_ESIZE otherwise).  No
 * entry point here allocates; calls that overlap on one GPU share the
 * scratch and race, so keep them in one stream (or serialise them). */
GRINQH_API int grinqh_calibrate_noalloc(const grinqh_layer_desc* desc, const void* x, int32_t S,
                                        const int32_t* p_bp, float* theta, void* stream);

/* Per-token precision assignment (Sec. 3.1; App. A.1).
 *   x: fp16 [B][K] (device), finite.
 *   mode GRINQH_ASSIGN_THRESHOLD: thresholds = host fp32 theta_1..theta_n
 *     (exactly n = n_levels-1 entries are read), non-decreasing, not NaN
 *     (+inf allowed); channel k gets the level l with |x_k| in
 *     [theta_l, theta_{l+1}), theta_0 = 0, theta_{n+1} = +inf, |x| compared
 *     in fp32.  counts = NULL.
 *   mode GRINQH_ASSIGN_TOPK: counts = host int32 c_0..c_n (exactly n_levels
 *     entries are read) summing to K (e.g. from grinqh_topk_counts).
 *     Channels are ordered by |x| descending, ties by lower index; the first
 *     c_n get level n, the next c_{n-1} level n-1, and so on.
 *     thresholds = NULL.  Requires K <= 16384.
 *   level_map: uint8 [B][K] (device), the level index per channel. */
GRINQH_API int grinqh_assign(const grinqh_layer_desc* desc, int mode, const void* x, int32_t B,
                  const float* thresholds, const int32_t* counts, uint8_t* level_map,
                  void* workspace, size_t ws_bytes, void* stream);

/* Nested-precision decode VMM (Sec. 3.3 reconstruction; App. C.1).
 *   y[t][n] = sum_k x[t][k] * w_hat(k, n), with w_hat = s*(q_b*2^(b_max-b)
 *   + phi - 2^(b_max-1)) for the b = level_bits[level_map[t][k]] most
 *   significant bits q_b of the code, phi = 2^(b_max-b-1) for 0 < b < b_max,
 *   phi = 0 at b = b_max, and channels at level 0 skipped.  Only the first b*T/8 bytes of each of a channel's
 *   rows are read; for B > 1 the deepest level over the B tokens is read once
 *   and each token uses its own prefix of it.
 *   x: fp16 [B][K]; level_map: uint8 [B][K], values < n_levels (a larger
 *   value is read as the top level); y: fp32 [B][N]; 1 <= B <= 4.
 *   flags: 0 -> y is overwritten (cleared by one extra launch before the
 *   VMM, whose workgroups add their partial sums into y); GRINQH_VMM_ACCUMULATE
 *   -> y += result (the caller initialised y, e.g. once for many VMMs into
 *   one buffer).  Accumulation order across K is not fixed, so y is
 *   reproducible to rounding, not bit for bit.  Any other flag bit is
 *   GRINQH_EINVAL.
 *   Precision: products and sums are at least those of fp32.  The matrix-core
 *   kernel holds each group's x in fixed point, 24 bits (23 for 1-bit planes)
 *   at the group's largest active |x|: a channel is exact down to 2^-13
 *   (2^-12) of that, and what the group's smaller channels lose together is at
 *   most 2^-22 (2^-21) of it. */
GRINQH_API int grinqh_vmm(const grinqh_layer_desc* desc, const void* packed_codes,
               const void* packed_scales, const void* x, const uint8_t* level_map,
               int32_t B, float* y, int32_t flags, void* workspace, size_t ws_bytes,
               void* stream);

/* The VMM with the threshold assignment of Sec. 3.1 fused into it: each
 * channel's level is graded inside the kernel from |x| and `thresholds`
 * (host fp32 theta_1..theta_n, rules as in grinqh_assign), so no level map
 * is read; if level_map_out is not NULL the levels are also written there
 * (uint8 [B][K]).  Other arguments as grinqh_vmm. */
GRINQH_API int grinqh_vmm_threshold(const grinqh_layer_desc* desc, const void* packed_codes,
                         const void* packed_scales, const void* x, int32_t B,
                         const float* thresholds, uint8_t* level_map_out, float* y,
                         int32_t flags, void* workspace, size_t ws_bytes, void* stream);

/* The batch-1 VMM with the exact top-k assignment of App. A.1 fused into
 * it: every workgroup selects the token's per-level cuts from the whole x
 * (the counts[j] channels of largest |x| at level j from the top, ties to the
 * lower channel index, exactly as grinqh_assign in top-k mode) and grades its
 * own channels against them, so no level map is read and no assignment
 * launch is needed.  counts: int32 [n_levels] (host), summing to K.
 * Requires B = 1, K <= 16384, 2-bit planes with tile_n in {256, 512, 1024}
 * (GRINQH_EUNSUPPORTED otherwise: grinqh_assign + grinqh_vmm serve the
 * other cases) and x 16-byte aligned.  level_map_out, if not NULL, receives
 * the levels (uint8 [K]).  Other arguments as grinqh_vmm.
 * Every workgroup repeats the selection, so on Llama3-8B-sized layers this
 * is slower than grinqh_assign (top-k) followed by grinqh_vmm; it serves
 * callers that cannot keep a level map or launch the assignment apart. */
GRINQH_API int grinqh_vmm_topk(const grinqh_layer_desc* desc, const void* packed_codes,
                               const void* packed_scales, const void* x, int32_t B,
                               const int32_t* counts, uint8_t* level_map_out, float* y,
                               int32_t flags, void* workspace, size_t ws_bytes, void* stream);

/* Prefill, the stage-decoupled dense path (Sec. 3: prefill reads the weights
 * at the fixed top precision; Sec. 4 "Prefill vs. Decoding Evaluation"): for
 * M tokens at once, every channel at all b_max bits,
 *   Y[m][n] = sum_k X[m][k] * w_hat[n][k],  w_hat = s[k/128][n] * (q[n][k] - 2^(b_max-1)),
 * with each w_hat rounded once to fp16 (the dequantised weight of a dense
 * fp16 GEMM), fp16 x fp16 products and fp32 accumulation: per element
 * |Y - exact| <= (2^-11 + K 2^-24) sum_k |X[m][k]| |w_hat[n][k]|.  Reads the
 * same packed buffers as grinqh_vmm (any plane_bits and tile_n).
 *   x: fp16 [M][K] (device, 16-byte aligned), finite; y: fp32 [M][N]
 *   (device, 4-byte aligned); 1 <= M <= 2^24.
 *   flags: 0 -> y is overwritten; GRINQH_VMM_ACCUMULATE -> y += result.
 * The summation order is fixed, so a result is reproducible bit for bit, and
 * accumulating adds to y exactly what overwriting would store in it. */
GRINQH_API int grinqh_prefill(const grinqh_layer_desc* desc, const void* packed_codes,
                              const void* packed_scales, const void* x, int32_t M, float* y,
                              int32_t flags, void* stream);

/* Infrastructure, not an operation of the paper: number of fp16 table
 * entries of a layer's look-up tables (host only), N * sum over levels
 * l >= 1 of 2^b_l. */
GRINQH_API int grinqh_lut_entries(const grinqh_layer_desc* desc, size_t* entries);

/* Decode VMM over non-uniform nested weights read through look-up tables
 * (Sec. 3.3: any quantiser with the nested property, e.g. nested k-means
 * weights, whose levels are centred so no midpoint bias applies; appendix
 * on nested weight formats).  Codes are packed as for grinqh_vmm (codes
 * source, no scales).
 *   luts: fp16, for each level l = 1..n (b = b_l bits) a table [N][2^b],
 *   the tables consecutive in level order: level l's table starts at
 *   element N * sum_{1 <= i < l} 2^b_i (16-byte aligned base).
 *   y[t][n] = sum_k x[t][k] * luts_l[n][q_b], l = level_map[t][k] (a value
 *   >= n_levels is read as the top level), q_b = the b leading bits of the
 *   b_max-bit code; level 0 skipped.
 *   x: fp16 [B][K]; level_map: uint8 [B][K]; y: fp32 [B][N]; 1 <= B <= 65535.
 *   flags: 0 -> y is overwritten; GRINQH_VMM_ACCUMULATE -> y += result.
 *   Partial sums meet in atomics: reproducible to rounding, not bit for bit. */
GRINQH_API int grinqh_vmm_lut(const grinqh_layer_desc* desc, const void* packed_codes,
                              const void* luts, const void* x, const uint8_t* level_map,
                              int32_t B, float* y, int32_t flags, void* stream);

/* The LUT VMM with the threshold assignment of Sec. 3.1 fused into it: each
 * channel's level is graded inside the kernel from |x| and `thresholds`
 * (host fp32 theta_1..theta_n, rules as in grinqh_assign), so no level map
 * is read; if level_map_out is not NULL the levels are also written there
 * (uint8 [B][K], device).  Other arguments as grinqh_vmm_lut. */
GRINQH_API int grinqh_vmm_lut_threshold(const grinqh_layer_desc* desc, const void* packed_codes,
                                        const void* luts, const void* x, int32_t B,
                                        const float* thresholds, uint8_t* level_map_out, float* y,
                                        int32_t flags, void* stream);

/* ------------------------------------------------------------------------
 * The key/value cache and the attention that reads it: what a decoder layer
 * does between its qkv and o projections.  Not part of the paper's method;
 * conventions (device memory, streams, validation, errors) as above.
 *
 * Cache layout.  K and V each have one array of pages.  A page holds `page`
 * consecutive tokens of one sequence, for every kv head:
 *   values [n_pages][heads][page][head_dim]  in the format's type (GRINQH_KV_I4: head_dim / 2 bytes)
 *   scales [n_pages][heads][page]            fp32, GRINQH_KV_I8
 *          [n_pages][heads][page][head_dim / 32][2]  fp16, GRINQH_KV_I4: step and base
 * GRINQH_KV_I8 holds a head of a token as int8 codes and one scale, the value
 * being code * scale (fp32).  With a = max|x| over the head_dim values of the
 * row in fp32: scale = fp32(a / 127), r = fp32(127 / a), code = rne(fp32(x * r)).
 * A row with a < 2^-100 is stored as zeros with scale 0; a row with a NaN or
 * an infinity as zeros with a NaN scale, so whatever reads it is NaN.
 * GRINQH_KV_I4 holds 32 channels at a time as codes 0..15 over their range, with
 * an fp16 step and base: base = fp16(min x), step = fp16(fp32((max x - base) / 15)),
 * 0 where that is negative, code = rne(fp32(fp32(x - base) / step)) clamped to 0..15,
 * 0 where the step is.  The value is code * step + base, rounded once to fp16.  A
 * group with a NaN, an infinity or a magnitude over 2^15 is stored as codes 0, step
 * 0 and a NaN base.  Channels 8 w .. 8 w + 7 are the little-endian 32-bit word w of a
 * row: channel 8 w + 2 i in bits 4 i .. 4 i + 3, channel 8 w + 2 i + 1 in bits
 * 16 + 4 i .. 16 + 4 i + 3.
 *
 * A batch is B sequences.  Row i of the n = row_offsets[b+1] - row_offsets[b]
 * rows of sequence b stands at position seq_lens[b] - n + i: the rows are the
 * last n tokens of the sequence (seq_lens counts them).  Token t of sequence b
 * is in place t % page of page block_table[b][t / page].
 * The batch's arrays live on the device and are read by the kernels, so a
 * captured graph follows what later steps write there.  What the host cannot
 * check is bounded in the kernels: offsets are clamped to 0..rows, a sequence
 * that ends before it starts has no rows, lengths are clamped to
 * 0..min(table_width * page, 2^30); rows of no sequence are not touched; memory
 * of a page id outside 0..n_pages-1 is never accessed.  Offsets have to ascend:
 * where they do not, nothing outside the arrays is touched, but which of the
 * rows between are done, and for which sequence, is not defined. */
enum { GRINQH_F16 = 0, GRINQH_BF16 = 1, GRINQH_F32 = 2 };            /* types of dense rows */
enum { GRINQH_KV_F16 = 0, GRINQH_KV_BF16 = 1, GRINQH_KV_I8 = 2,      /* formats of the cache */
       GRINQH_KV_I4 = 4 };

typedef struct {
  int32_t format;    /* GRINQH_KV_* */
  int32_t heads;     /* kv heads, 1..1024 */
  int32_t head_dim;  /* 64 or 128 */
  int32_t page;      /* tokens per page, a power of two, 1..2^20 */
  int32_t n_pages;   /* pages of the arrays, >= 1 */
} grinqh_kv_desc;

typedef struct {
  void* k;           /* device, 16-byte aligned */
  void* v;
  void* k_scale;     /* device, 4-byte aligned; NULL for 16-bit formats */
  void* v_scale;
} grinqh_kv_cache;

typedef struct {
  const int32_t* block_table;  /* device [B][table_width]: page ids */
  const int32_t* seq_lens;     /* device [B]: tokens of each sequence, its rows included */
  const int32_t* row_offsets;  /* device [B + 1]: where each sequence's rows start */
  int32_t B;                   /* sequences, 0..65535 */
  int32_t table_width;         /* page ids per sequence, >= 1 */
  int32_t rows;                /* rows of the dense arrays, 0..2^24; in attention times the
                                  query heads at most 2^30 */
} grinqh_kv_batch;

/* Dense rows [rows][heads][head_dim]: the last axis contiguous, the others with
 * strides in elements, 0..2^36 and multiples of 16 bytes; base 16-byte aligned.
 * Rows that are written must not overlap. */
typedef struct {
  void* data;
  int64_t row_stride;
  int64_t head_stride;
} grinqh_rows;

/* Sizes of the arrays of K (those of V are the same): value bytes and scale
 * bytes (0 for 16-bit formats).  Host only. */
GRINQH_API int grinqh_kv_bytes(const grinqh_kv_desc* desc, size_t* value_bytes, size_t* scale_bytes);

/* Write the batch's rows of K and V (type GRINQH_F16, GRINQH_BF16 or
 * GRINQH_F32) into the cache, quantised as the format asks; 16-bit formats
 * round to nearest even.  A row is not written if its position is negative or
 * its page id out of range.  Where two rows share a slot either may stay. */
GRINQH_API int grinqh_kv_write(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache,
                               const grinqh_kv_batch* batch, int type, const grinqh_rows* k,
                               const grinqh_rows* v, void* stream);

/* Read the batch's rows back from the cache as dense K and V of `type`
 * (rounded to nearest even; offsets = the running sum of seq_lens reads whole
 * sequences).  A row whose position is negative is zeros, one whose page id is
 * out of range NaN. */
GRINQH_API int grinqh_kv_read(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache,
                              const grinqh_kv_batch* batch, int type, const grinqh_rows* k,
                              const grinqh_rows* v, void* stream);

typedef struct {
  int32_t heads;     /* query heads, a multiple of the cache's; kv head h serves query heads
                        h * heads / kv_heads onwards */
  int32_t type;      /* of q and out: GRINQH_F16 or GRINQH_BF16; a 16-bit cache has the same */
  float scale;       /* of the scores; positive and finite (usually head_dim^-1/2) */
  int32_t window;    /* 0: every earlier token is visible; W > 0: the row's own and the W - 1
                        tokens before it */
  int32_t sinks;     /* first tokens of a sequence that stay visible behind the window */
  int32_t max_rows;  /* upper estimates of the rows and of the length of one sequence: they
                        shape the launch and never change what is computed.  Loose ones
                        cost time: 32 tokens decoded after up to 8190 others take 66 us with
                        exact ones, 193 us with max_len = 131072, 387 us with max_rows = 32 */
  int32_t max_len;
} grinqh_attend_desc;

/* Attention of the batch's rows over the cache.  The row at position p sees
 * token t iff t <= p and (window = 0 or t > p - window or t < sinks), with
 *   s_t = scale * (q . k_t), m = max s_t, o = sum_t exp(s_t - m) v_t / sum_t exp(s_t - m)
 * over the visible t.  A row that sees nothing (or only scores of -inf) is 0.
 * lse (fp32 [rows][heads], contiguous, or NULL) gets m + log sum_t exp(s_t - m),
 * -inf for such a row.  What a row does not see never reaches it, infinities
 * and NaN included; a value that it sees and that is not finite makes its
 * channel infinite or NaN; a visible token whose page id is out of range makes the
 * row NaN, pages that no row sees may have any id.
 * Precision: scores, statistics and sums in fp32; a 4-bit cache's values are
 * fp16, and are read as an fp16 cache's; exp(s_t - m), at an 8-bit
 * cache times the value's scale, is rounded to 16 bits for the product with
 * the values (fp16, for a bf16 cache bf16).  In fp16 11 bits of it stay down
 * to 2^-23 of the row's largest weight, at an 8-bit cache to value scales 2^23
 * below the largest that the row has seen; what is below is off by at most
 * 2^-34 (2^-33 at 8 bits) of the largest.  Scores times log2 e have to stay
 * inside fp32; of bf16 queries over an 8- or 4-bit cache, which are held as fp16
 * times a power of two, (q . k) / max |q| has to stay under 2^112.
 * The rows' own tokens have to be in the cache already (grinqh_kv_write).
 * workspace: device, 16-byte aligned, of at least the size that
 * grinqh_attend_workspace_bytes gives for the same arguments (host only; may
 * be 0: NULL).  It holds partial results of sequences that are split over
 * workgroups; calls on different streams need workspaces of their own. */
GRINQH_API int grinqh_attend_workspace_bytes(const grinqh_kv_desc* desc, const grinqh_attend_desc* attend,
                                             int32_t B, int32_t rows, size_t* bytes);
GRINQH_API int grinqh_attend(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache,
                             const grinqh_kv_batch* batch, const grinqh_attend_desc* attend,
                             const grinqh_rows* q, const grinqh_rows* out, float* lse,
                             void* workspace, size_t ws_bytes, void* stream);

/* Planning a step: the arrays of a batch, and the cache's pages, follow the
 * tokens that come to each sequence or are taken back.  The pages that no
 * sequence holds stand in a list on the device, the next one to be handed out
 * last. */
typedef struct {
  int32_t* free_pages;  /* device [capacity]; the first n_free are ids of free pages */
  int32_t* n_free;      /* device [1]; read as 0..capacity */
  int32_t capacity;     /* 1..2^30 */
} grinqh_kv_pool;

/* One step of B sequences.  new_rows[b] > 0: that many tokens come to sequence
 * b; < 0: that many of its last tokens are taken back (all of them, if it has
 * fewer); 0: neither.  In this order:
 *   Tokens taken back.  seq_lens[b] falls; pages that hold none of the sequence's
 *   tokens any more go to the list, their table entries become -1.  An entry out
 *   of range (0..n_pages-1) is no page and does not go there.  The pages stand in
 *   the list so that the first sequence's first page is the next to be handed
 *   out.  Pages past the list's capacity are lost.
 *   Tokens that come.  A sequence asks for new_rows[b] rows and for the pages
 *   that its new length takes beyond the old one.  Where the new length passes
 *   min(table_width * page, 2^30) it gets nothing.  Of the others, in order, each
 *   gets what it asks for as long as the running sums of the pages and of the
 *   rows, its own included, do not pass the list's pages and `rows`; from the
 *   first that does on, none gets anything.  seq_lens[b] rises, pages leave the
 *   list from its end into the sequence's table entries.
 * row_offsets [B + 1] are written: the running sum of the rows that come, which
 * are the last tokens of their sequences, as grinqh_kv_write and grinqh_attend
 * expect them.  Optional (NULL), for the caller's own kernels, as nothing here reads
 * them: positions [rows], the position of each row in its sequence (a rotary
 * embedding's); slots [rows], page id * page + place in the page, or -1 for a page
 * id out of range; both are -1 behind the last row; granted [B]: new_rows[b], 0
 * where nothing was given, minus the tokens that were taken back.
 * seq_lens are read as 0..min(table_width * page, 2^30).  A sequence's pages are its own:
 * one that stands in two tables would go to the list twice.  Everything but
 * desc, B, table_width, rows and the addresses is read on the device, so a
 * captured graph follows it.  The arrays must not overlap.  B = 0..65535, rows =
 * 0..2^24.  workspace: device, 16-byte aligned, of the size that
 * grinqh_kv_plan_workspace_bytes gives for B (host only); calls on different
 * streams need workspaces of their own.  Results do not depend on the order in
 * which workgroups run. */
GRINQH_API int grinqh_kv_plan_workspace_bytes(int32_t B, size_t* bytes);
GRINQH_API int grinqh_kv_plan(const grinqh_kv_desc* desc, const grinqh_kv_pool* pool, int32_t B, int32_t table_width,
                              int32_t rows, const int32_t* new_rows, int32_t* block_table, int32_t* seq_lens,
                              int32_t* row_offsets, int32_t* positions, int64_t* slots, int32_t* granted,
                              void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Between the blocks of a layer: norms, gate and residual stream.  Not part of the
 * paper's method; conventions as above.
 *   a  = post(y), of the block's output y             (post: a norm or none)
 *   h' = residual_scale * h + gate * a                (gate per channel, or per row and channel)
 *   x  = pre(h'), what the next block reads           (pre: a norm or none)
 * over rows of n channels, with the norms
 *   GRINQH_NORM_RMS    v / sqrt(mean(v^2) + eps) * weight + bias
 *   GRINQH_NORM_LAYER  (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * weight + bias
 * All in fp32; h_out and x are rounded once, x from the h' that is not rounded.
 * A norm's squares and sums may leave fp32's range; a, gate * a, h' and the results
 * have to be in it.  A row of one value has a LAYER norm of its bias, however far
 * that value is from zero; with eps = 0 it is NaN, as a row of zeros is in either. */
enum { GRINQH_NORM_NONE = 0, GRINQH_NORM_RMS = 1, GRINQH_NORM_LAYER = 2 };

typedef struct {
  int32_t rows;             /* 0..2^24 */
  int32_t n;                /* channels, 1..32768 */
  int32_t post, pre;        /* GRINQH_NORM_* */
  int32_t y_type, h_type, x_type, gate_type, weight_type;  /* GRINQH_F16, GRINQH_BF16 or GRINQH_F32 */
  float residual_scale;     /* finite */
  float eps;                /* of both norms; finite, not negative */
} grinqh_norm_desc;

/* Device arrays, aligned to their elements; strides of rows in elements, n..2^36
 * (inputs: 0 too, one row for all).  NULL: y (a = 0), h (no residual stream), gate
 * (1), weights (1), biases (0), h_out and x (not wanted), but not both y and h,
 * nor both h_out and x; x is wanted only with a pre norm.  Without a post norm
 * its weight and bias must be NULL, as without a pre norm that one's.  h_out may
 * be h or y, x may be y (if h_out is not), where type and stride are the same; else
 * what is written must not overlap anything.  With rows = 0 they are not looked at. */
typedef struct {
  const void* y;    int64_t y_stride;
  const void* h;    int64_t h_stride;
  const void* gate; int64_t gate_stride;
  void* h_out;      int64_t h_out_stride;
  void* x;          int64_t x_stride;
  const void *post_weight, *post_bias, *weight, *bias;   /* [n] of weight_type */
} grinqh_norm_arrays;

GRINQH_API int grinqh_norm(const grinqh_norm_desc* desc, const grinqh_norm_arrays* arrays, void* stream);

/* Infrastructure for tests and measurements, not an operation of the paper:
 * process-wide overrides of launch choices that never change results beyond
 * rounding order.  Value 0 restores each launcher's own choice.
 *   GRINQH_OPT_VMM_KERNEL: GRINQH_KERNEL_PER_PLANE or GRINQH_KERNEL_GENERAL
 *     runs that kernel (grinqh_vmm, grinqh_vmm_threshold, any B) in place of
 *     the default ones.
 *   GRINQH_OPT_GROUPS_PER_WG: chooses between the two default kernels at B = 1
 *     and 2-bit planes: 1 the matrix-core kernel (one group of 128 channels per
 *     workgroup), 2..4 the register kernel (two groups).  The per-plane kernel
 *     takes that many groups per workgroup, or its maximum if that is less.
 *   GRINQH_OPT_PREFILL_TILE: 1, 2, 3 = 256x256, 256x128, 128x128 prefill tiles.
 *   GRINQH_OPT_LUT_GROUPS: 1..16 groups per workgroup of the LUT VMM.
 *   GRINQH_OPT_PREFILL_CUS: 1..4096, the CU count the prefill balances its
 *     rounds of 256x256 tiles for (0: the device's).
 *   GRINQH_OPT_ATTEND_KERNEL: GRINQH_ATTEND_ROWS (16 or 32 rows per workgroup)
 *     or GRINQH_ATTEND_TILE (256); GRINQH_OPT_ATTEND_SPLITS: 1..1024 parts of
 *     a sequence's tokens.  grinqh_attend_workspace_bytes
 *     follows both, so set them before asking for the size.
 * Returns GRINQH_EINVAL for an unknown option or a value out of range.  The
 * setting is read when a call enqueues its kernels; set it between calls. */
GRINQH_API int grinqh_set_option(int option, int value);

/* Measurement infrastructure, not an operation of the paper: read `bytes` of
 * device memory at src (16-byte aligned; a positive multiple of 2 MiB) with
 * non-temporal 16-byte loads, eight in flight per lane, as fast as the chip
 * streams them, and XOR a fold of the data into *sink (device uint32).  It
 * gives the measured streaming-read ceiling the VMM's bandwidth is compared
 * with. */
GRINQH_API int grinqh_stream_read(const void* src, size_t bytes, uint32_t* sink, void* stream);

/* Infrastructure, not an operation of the paper: the message of the last
 * failing call on this thread ("" if none), valid until that thread's next
 * call. */
GRINQH_API const char* grinqh_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* GRINQH_H */
