/*
 * sq.h -- C ABI of the MI355X (gfx950) rotated W4A4 inference path of SpinQuant
 * (arXiv 2405.16406): online Hadamard rotation + 4-bit activation quantization, offline
 * weight preparation, the int4 x int4 GEMM with its dequantising epilogue, and R3 +
 * 4-bit KV-cache quantization.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Pointers named "device" are HIP device pointers (or memory the device can read
 *    and write).  The caller allocates and owns every buffer, keeps it alive until
 *    the enqueued work has finished, and synchronises.  The library never allocates,
 *    frees or synchronises; it only enqueues kernels on `stream` (a hipStream_t; NULL
 *    means the default stream).  Calls are asynchronous.
 *  - Tensors are row-major.  fp16 is IEEE binary16; scales are fp32.
 *  - 4-bit codes are packed two per byte along the row, the element with the even
 *    index in the low nibble.  Activation and KV codes are unsigned (0..15); weight
 *    codes are two's-complement nibbles (-7..7).
 *  - Quantization follows eq. 1 of the paper (Sec. 2):
 *        X_Q = alpha * round((X - beta) / alpha) + beta,
 *    asymmetric (alpha = (max-min)/(2^N-1), beta = min) for activations and the KV
 *    cache, symmetric (alpha = max|X|/(2^(N-1)-1), beta = 0) for weights, no range
 *    clipping (App. A, "Quantization choice", Table 12).  Round-to-nearest is ties to
 *    even; (X-beta)/alpha is evaluated as (X-beta) * fl32(1/alpha); a group whose
 *    alpha would be zero or subnormal (e.g. a constant group) gets alpha = 1, codes 0.
 *  - Online rotation (R4 on the down-projection input, R3 on Q/K; Sec. 3.1
 *    "Additional unabsorbed rotations"): each contiguous block of n = a*b elements of
 *    a row is multiplied on the right by R = (H_a (x) S_b) / sqrt(n), where H_a is a
 *    +-1 Hadamard matrix of order a and S_b the natural-order Sylvester matrix of order
 *    b = 2^k (dense factor on the outer, strided index: element i = i_a*b + i_b).
 *    (a, b) = (1, 1) is the identity.
 *  - Errors: every argument is checked on the host before anything is enqueued.  A
 *    non-OK status means nothing was enqueued and no output was written; the message
 *    is available from sq_last_error() (per thread).  Launch failures, including "no
 *    device", return SQ_ERR_HIP.  Arguments are never dereferenced on the host.
 */
#ifndef SQ_H_
#define SQ_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SQ_ABI_VERSION 1

/* Largest row length K accepted by sq_had_quant_act / sq_pack_w4 (rotated or not). */
#define SQ_MAX_ROW 32768
/* Largest dense Hadamard factor order a. */
#define SQ_MAX_DENSE 256

typedef enum {
  SQ_OK = 0,
  SQ_ERR_NULL = 1,        /* a required pointer is NULL */
  SQ_ERR_SHAPE = 2,       /* sizes inconsistent or out of range */
  SQ_ERR_UNSUPPORTED = 3, /* a valid request the library does not implement (e.g. bits = 6) */
  SQ_ERR_ALIGN = 4,       /* pointer or leading dimension misaligned */
  SQ_ERR_ALIAS = 5,       /* an output overlaps an input or another output */
  SQ_ERR_HIP = 6          /* the HIP runtime reported an error (no device, launch failure) */
} sq_status;

/* SQ_ABI_VERSION of the built library. */
int32_t sq_abi_version(void);

/* Message for the last non-OK status returned on the calling thread ("" if none). */
const char* sq_last_error(void);

/*
 * sq_time_next_call -- measurement hook, not part of the method.  Arms two events for
 * the next call of sq_had_quant_act(_ex), sq_pack_w4(_ex), sq_w4a4_linear, sq_w4a8_linear,
 * sq_w4a4_linear_swiglu, sq_qk_had_kvquant(_ex), sq_attn_decode_kv4(_ex),
 * sq_rope_kv_write(_ex), sq_kv_read, sq_attn_paged(_window), sq_attn_prompt(_window), sq_attn_tree,
 * sq_tree_mask, sq_paged_release, sq_paged_grow or sq_kv_keep made by this host thread:
 * start_event takes the start time of the first kernel that call launches and stop_event
 * the end time of its last kernel (hipExtLaunchKernel events), so hipEventElapsedTime(start,
 * stop) is the call's time on the device without marker packets between kernels.
 *   start_event, stop_event   hipEvent_t, created by the caller with timing enabled
 * The events are consumed by that next call whatever its outcome; a call that returns
 * an error, or enqueues nothing (M == 0), leaves them as they were.
 * Errors: SQ_ERR_NULL for a NULL event.
 */
sq_status sq_time_next_call(void* start_event, void* stop_event);

/*
 * sq_hadamard_factor -- host helper: writes the library's +-1 Hadamard matrix of order
 * n into out_host[n*n] (row-major int8, HOST memory), for use as `had_dense`.
 *   n = 1    : [1]
 *   n = 28   : Paley type II construction from q = 13
 *   n = 172  : Williamson construction from four symmetric circulants of order 43
 * Any Hadamard matrix is a valid rotation factor (Sec. 3.1 only asks for "a Hadamard
 * matrix"); these are the ones the library provides.  Errors: SQ_ERR_NULL,
 * SQ_ERR_UNSUPPORTED (other n).
 */
sq_status sq_hadamard_factor(int32_t n, int8_t* out_host);

/*
 * sq_had_quant_act -- online Hadamard rotation of every activation row (R4, Sec. 3.1) fused with asymmetric 4-bit quantization of
 * eq. 1 (Sec. 2) and nibble packing, or 8-bit quantization (the W4A8 setting, Sec. 4.2).
 *
 *   x          device fp16 [M, ldx], row stride ldx elements; row m is x[m*ldx .. +K)
 *   M, K       rows (tokens) and row length; M >= 0 (M == 0 is a no-op), 0 < K <= SQ_MAX_ROW,
 *              K % 8 == 0
 *   ldx        >= K, ldx % 8 == 0; x must be 16-byte aligned
 *   had_dense_n  a, order of the dense factor, 1 <= a <= SQ_MAX_DENSE
 *   had_dense  device int8 +-1 [a, a] row-major (must be a Hadamard matrix); NULL iff a == 1
 *   had_pow2_n b, power of two, 1 <= b <= 32768; n = a*b must divide K
 *   bits       4 or 8 (others: SQ_ERR_UNSUPPORTED)
 *   group      quantization group length along the row: group | K, group % 2 == 0;
 *              group == K is per-token quantization (what sq_w4a4_linear consumes)
 *   q_out      device uint8, 16-byte aligned, contiguous: bits 4: [M, K/2] packed codes
 *              0..15 (even k in the low nibble); bits 8: [M, K] codes 0..255
 *   alpha, beta device fp32 [M, K/group] (contiguous): scale and offset of each group
 *   dbg_rot    optional device fp32 [M, K]: the rotated rows (quantizer input); NULL to skip
 *   stream     hipStream_t
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_had_quant_act(const void* x, int64_t M, int64_t K, int64_t ldx,
                           int32_t had_dense_n, const int8_t* had_dense, int32_t had_pow2_n,
                           int32_t bits, int32_t group,
                           uint8_t* q_out, float* alpha, float* beta, float* dbg_rot,
                           void* stream);

/*
 * sq_had_quant_act_ex -- sq_had_quant_act with the two variants the paper compares its
 * choices against (sq_had_quant_act is this call with signs = NULL and clip = 1):
 *   signs      optional device int8 [a*b] (a = had_dense_n, b = had_pow2_n): the diagonal
 *              S of a random Hadamard matrix S H (Sec. 2.2), so that each block of n = a*b
 *              elements is multiplied by S (H_a (x) S_b) / sqrt(n); element i of a block is
 *              multiplied by signs[i] first.  Entries are +1 or -1 (only their sign is read:
 *              negative = -1).  NULL for none.  Any alignment.
 *   clip       range clipping ratio r, 0 < r <= 1 (App. A "Quantization choice"): each group
 *              is quantized over [r min, r max] (each end rounded to fp32), so
 *              alpha = fl(fl(r max) - fl(r min)) / L, beta = fl(r min), and codes of values
 *              outside the range clamp to 0 or L.  1 is plain min-max.
 *              Outside (0, 1] (NaN included): SQ_ERR_SHAPE.
 * Every other argument, layout and error as sq_had_quant_act; signs is an input for the
 * overlap check.
 */
sq_status sq_had_quant_act_ex(const void* x, int64_t M, int64_t K, int64_t ldx,
                              int32_t had_dense_n, const int8_t* had_dense, int32_t had_pow2_n,
                              const int8_t* signs, int32_t bits, int32_t group, float clip,
                              uint8_t* q_out, float* alpha, float* beta, float* dbg_rot,
                              void* stream);

/*
 * sq_pack_w4 -- offline weight preparation: optionally absorb the online
 * rotation into the weight, W' = W R (Sec. 3.1: rotations merge into the adjacent
 * weights, so (x R)(W R)^T = x W^T), then symmetric 4-bit quantization of eq. 1 per
 * output channel (row), nibble packing, and the per-row sum of codes used by the
 * epilogue's zero-point term.
 *
 *   w          device fp16 [N, ldw], 16-byte aligned, ldw >= K, ldw % 8 == 0
 *   N, K       output channels and row length; N >= 0, 0 < K <= SQ_MAX_ROW, K % 8 == 0
 *   had_dense_n, had_dense, had_pow2_n   rotation as in sq_had_quant_act ((1, NULL, 1) = none)
 *   wq         device uint8 [N, K/2], 16-byte aligned: two's-complement nibbles -7..7
 *   w_alpha    device fp32 [N]: per-channel scale
 *   w_rowsum   device int32 [N]: sum over k of the codes of row n
 * Errors: as sq_had_quant_act.
 */
sq_status sq_pack_w4(const void* w, int64_t N, int64_t K, int64_t ldw,
                     int32_t had_dense_n, const int8_t* had_dense, int32_t had_pow2_n,
                     uint8_t* wq, float* w_alpha, int32_t* w_rowsum, void* stream);

/*
 * sq_pack_w4_ex -- sq_pack_w4 absorbing the random Hadamard rotation S H of Sec. 2.2:
 * W' = W R with R = S (H_a (x) S_b) / sqrt(n) blockwise, the same R that
 * sq_had_quant_act_ex applies to the activations with the same signs, so that
 * (x R)(W R)^T = x W^T.
 *   signs      optional device int8 [a*b], +1 or -1 (sign read), as in sq_had_quant_act_ex;
 *              NULL makes this call sq_pack_w4
 * Every other argument, layout and error as sq_pack_w4.
 */
sq_status sq_pack_w4_ex(const void* w, int64_t N, int64_t K, int64_t ldw,
                        int32_t had_dense_n, const int8_t* had_dense, int32_t had_pow2_n, const int8_t* signs,
                        uint8_t* wq, float* w_alpha, int32_t* w_rowsum, void* stream);

/*
 * sq_w4a4_linear -- the quantized linear layer y = x W^T on 4-bit codes.  The int4 x int4 products
 * accumulate exactly in int32, acc[m,n] = sum_k qa[m,k] qw[n,k]; the epilogue expands
 * eq. 1 on both operands:
 *     y[m,n] = fp16( w_alpha[n] * (x_alpha[m] * acc[m,n] + x_beta[m] * w_rowsum[n]) + bias[n] )
 *
 *   xq         device uint8 [M, K/2], 16-byte aligned: per-token activation codes
 *              (from sq_had_quant_act with group == K)
 *   x_alpha, x_beta  device fp32 [M]
 *   M          >= 0 (0 is a no-op)
 *   wq, w_alpha, w_rowsum   device, from sq_pack_w4: uint8 [N, K/2] (16-byte aligned), fp32 [N], int32 [N]
 *   N          >= 1
 *   K          > 0, K % 64 == 0, K <= 2^20 (the int32 accumulator holds 16 x acc, and
 *              16 x 15 x 7 x 2^20 < 2^31)
 *   bias       optional device fp16 [N]; NULL for none
 *   y          device fp16 [M, ldy], ldy >= N, 2-byte aligned
 *   dbg_acc    optional device int32 [M, N] (contiguous): the raw accumulators; NULL to skip
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_w4a4_linear(const uint8_t* xq, const float* x_alpha, const float* x_beta, int64_t M,
                         const uint8_t* wq, const float* w_alpha, const int32_t* w_rowsum,
                         int64_t N, int64_t K, const void* bias, void* y, int64_t ldy,
                         int32_t* dbg_acc, void* stream);

/*
 * sq_w4a8_linear -- the quantized linear layer of the W4A8 setting (Sec. 4.2, 4.5): 8-bit
 * per-token activation codes (sq_had_quant_act with bits = 8, group = K) against the 4-bit
 * weights of sq_pack_w4.  acc[m,n] = sum_k qa[m,k] qw[n,k] exactly in int32 and
 *     y[m,n] = fp16( w_alpha[n] * (x_alpha[m] * acc[m,n] + x_beta[m] * w_rowsum[n]) + bias[n] )
 *
 *   xq         device uint8 [M, K] (contiguous), 16-byte aligned: codes 0..255
 *   x_alpha, x_beta, M, wq, w_alpha, w_rowsum, N, bias, y, ldy, dbg_acc   as for sq_w4a4_linear
 *   K          > 0, K % 64 == 0, K <= 2^17 (the int32 sums of 16 x (qa - 128) x qw)
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_w4a8_linear(const uint8_t* xq, const float* x_alpha, const float* x_beta, int64_t M,
                         const uint8_t* wq, const float* w_alpha, const int32_t* w_rowsum,
                         int64_t N, int64_t K, const void* bias, void* y, int64_t ldy,
                         int32_t* dbg_acc, void* stream);

/*
 * sq_w4a4_linear_swiglu -- the gate and up projections of the MLP in one product, combined
 * in the epilogue into the input of down_proj, the activation that R4 rotates (Sec. 3.1,
 * Fig. 1(c)):
 *     h[m,c] = fp16( SiLU(g[m,c]) * u[m,c] ),  SiLU(v) = v / (1 + e^-v),
 * where g and u are the dequantised outputs of sq_w4a4_linear for the gate and up weights,
 * kept in fp32 (not rounded to fp16) before they are combined.
 *
 *   xq, x_alpha, x_beta, M, K, stream   as for sq_w4a4_linear (K <= 2^20)
 *   wq, w_alpha, w_rowsum, bias   the gate and up weights packed by sq_pack_w4 as one
 *              [N, K] matrix whose rows interleave them in blocks of 32: rows 64b .. 64b+31
 *              are gate rows 32b .. 32b+31 and rows 64b+32 .. 64b+63 the up rows of the
 *              same outputs (packing is per row, so this is the two matrices' packed rows
 *              reordered); bias (optional) in the same order
 *   N          2 * I (I outputs), N % 64 == 0
 *   h          device fp16 [M, ldh], ldh >= N/2, 2-byte aligned
 * No raw-accumulator output (sq_w4a4_linear gives the accumulators of the same product).
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_UNSUPPORTED (operands
 * of about 2^31 bytes and more: (M + 256) K/2 and (N + 256) K/2 below 2^31 - 128 are always
 * taken; with M <= 16 only the weights count, with M <= 2 and K <= 65536 nothing is refused),
 * SQ_ERR_HIP.
 */
sq_status sq_w4a4_linear_swiglu(const uint8_t* xq, const float* x_alpha, const float* x_beta, int64_t M,
                                const uint8_t* wq, const float* w_alpha, const int32_t* w_rowsum,
                                int64_t N, int64_t K, const void* bias, void* h, int64_t ldh, void* stream);

/*
 * sq_qk_had_kvquant -- R3 (Sec. 3.1) on post-RoPE queries and keys, per head,
 * R = S_D / sqrt(D); then asymmetric 4-bit (or 8-bit: KV8) quantization of eq. 1 of the rotated keys
 * and of the (unrotated) values, one group per `group` contiguous elements of a head
 * vector (group == D: one (alpha, beta) per batch, token and head).
 *
 *   q, k, v    device fp16 [B, S, H, D] contiguous, 16-byte aligned
 *   B, S, H    >= 0 (any zero: no-op); D = 128
 *   bits       4 or 8; group = 128 (= D)
 *   q_rot      device fp16 [B, S, H, D]: Q R, rounded to nearest fp16
 *   k_q, v_q   device uint8, 16-byte aligned: bits 4: [B, S, H, D/2] packed codes 0..15;
 *              bits 8: [B, S, H, D] codes 0..255
 *   k_alpha, k_beta, v_alpha, v_beta   device fp32 [B, S, H, D/group]
 *   dbg_k_rot  optional device fp32 [B, S, H, D]: K R before quantization; NULL to skip
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_qk_had_kvquant(const void* q, const void* k, const void* v,
                            int64_t B, int64_t S, int64_t H, int64_t D, int32_t bits, int32_t group,
                            void* q_rot, uint8_t* k_q, float* k_alpha, float* k_beta,
                            uint8_t* v_q, float* v_alpha, float* v_beta, float* dbg_k_rot,
                            void* stream);

/*
 * sq_qk_had_kvquant_ex -- sq_qk_had_kvquant with range clipping of the cache groups
 * (App. A "Quantization choice" compares clipped and unclipped KV quantizers) and an fp16
 * storage of the group parameters; sq_qk_had_kvquant is this call with k_clip = v_clip = 1
 * and param_bits = 32.
 *   k_clip, v_clip  clipping ratios r, 0 < r <= 1, of the key and value groups: a group is
 *              quantized over [r min, r max] (ends rounded to fp32; for keys the min and max
 *              of the rotated values), codes outside clamp to 0 or L.
 *              Outside (0, 1] (NaN included): SQ_ERR_SHAPE.
 *   param_bits 32: k_alpha, k_beta, v_alpha, v_beta are fp32 [B, S, H, D/group] (4-byte
 *              aligned); 16: fp16 of the same shape (2-byte aligned), half the parameter
 *              bytes of the cache.  fp16 parameters are the fp32 ones rounded to nearest even,
 *              saturated at +-65504; a group whose fp16 alpha is 0 is constant (alpha 1,
 *              codes 0); codes are then taken from the stored pair,
 *              c = clamp(rint((x - beta16) / alpha16), 0, L), each step rounded in fp32.
 *              Other values: SQ_ERR_UNSUPPORTED.
 * Every other argument, layout and error as sq_qk_had_kvquant.
 */
sq_status sq_qk_had_kvquant_ex(const void* q, const void* k, const void* v,
                               int64_t B, int64_t S, int64_t H, int64_t D, int32_t bits, int32_t group,
                               float k_clip, float v_clip, int32_t param_bits,
                               void* q_rot, uint8_t* k_q, void* k_alpha, void* k_beta,
                               uint8_t* v_q, void* v_alpha, void* v_beta, float* dbg_k_rot,
                               void* stream);

/*
 * sq_attn_decode_kv4 -- attention of one new query per (batch, head) over the 4-bit KV
 * cache written by sq_qk_had_kvquant, the step that consumes it.  Keys and values are
 * dequantised group by group with eq. 1, K_t = k_alpha_t * c_t + k_beta_t (in the R3-rotated
 * basis) and V_t likewise; the query is the R3-rotated one (q_rot of sq_qk_had_kvquant), so
 * q_rot . K_t is the score of the unrotated query and key (Sec. 3.1):
 *     out[b,h,:] = fp16( sum_t softmax_t(scale * q_rot[b,h,:] . K_t) V_t ),  t = 0 .. S-1.
 *
 *   q_rot      device fp16 [B, H, 128] (contiguous), 16-byte aligned
 *   k_q, v_q   device uint8 [B, S, H, 64] (the sq_qk_had_kvquant layout), 16-byte aligned
 *   k_alpha, k_beta, v_alpha, v_beta  device fp32 [B, S, H]
 *   B, S, H    B >= 0 (0 is a no-op), S >= 1, H >= 1, B * H < 2^31, S * H * 64 < 2^31
 *   D          128 (others: SQ_ERR_UNSUPPORTED)
 *   scale      finite score scale, e.g. 1/sqrt(128)
 *   out        device fp16 [B, H, 128] (contiguous), 16-byte aligned
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_attn_decode_kv4(const void* q_rot, const uint8_t* k_q, const float* k_alpha, const float* k_beta,
                             const uint8_t* v_q, const float* v_alpha, const float* v_beta,
                             int64_t B, int64_t S, int64_t H, int64_t D, float scale, void* out, void* stream);

/*
 * sq_attn_decode_kv4_ex -- sq_attn_decode_kv4 over a cache whose group parameters are stored
 * as written by sq_qk_had_kvquant_ex with the same param_bits (32: fp32, 16: fp16 [B, S, H],
 * aligned to their size); sq_attn_decode_kv4 is this call with param_bits = 32.
 * Other param_bits: SQ_ERR_UNSUPPORTED.  Every other argument, layout and error as
 * sq_attn_decode_kv4.
 */
sq_status sq_attn_decode_kv4_ex(const void* q_rot, const uint8_t* k_q, const void* k_alpha, const void* k_beta,
                                const uint8_t* v_q, const void* v_alpha, const void* v_beta,
                                int64_t B, int64_t S, int64_t H, int64_t D, float scale, int32_t param_bits,
                                void* out, void* stream);

/*
 * sq_attn_decode_workspace -- device bytes of the workspace sq_attn_decode_kv4_split needs
 * for B, S, H and D on the CURRENT device (the split depends on its compute-unit count):
 * B * H * chunks * 528, where chunks is the number of pieces the S tokens are split into
 * (0 bytes when they are not split).  Shape rules and errors of sq_attn_decode_kv4;
 * SQ_ERR_NULL for a NULL bytes; SQ_ERR_HIP when the device cannot be queried.
 */
sq_status sq_attn_decode_workspace(int64_t B, int64_t S, int64_t H, int64_t D, uint64_t* bytes);

/*
 * sq_attn_decode_kv4_split -- the attention of sq_attn_decode_kv4_ex (same formula, Sec. 3.1
 * R3 with eq. 1 dequantisation), split over the sequence as in flash-decoding: each
 * workgroup reads one chunk of tokens for 16 heads at once, 1 KB of one token per wave
 * load; a second kernel merges the chunks' partial softmax states (maximum, sum,
 * 128 weighted dims, in fp32) in chunk order.  The result equals sq_attn_decode_kv4_ex's
 * up to the order of fp32 additions, and is deterministic.
 *   workspace        device memory, 16-byte aligned, at least the bytes
 *                    sq_attn_decode_workspace gives (NULL allowed when that is 0); the
 *                    caller owns it; its contents need no initialisation and are scratch
 *                    after the call; it must not overlap any argument
 *   workspace_bytes  its size in bytes
 * Every other argument, layout and error as sq_attn_decode_kv4_ex; SQ_ERR_SHAPE when the
 * workspace is too small, SQ_ERR_ALIGN / SQ_ERR_ALIAS for its alignment and overlaps.
 * Calls that share a workspace must be ordered (same stream, or synchronised).
 */
sq_status sq_attn_decode_kv4_split(const void* q_rot, const uint8_t* k_q, const void* k_alpha, const void* k_beta,
                                   const uint8_t* v_q, const void* v_alpha, const void* v_beta,
                                   int64_t B, int64_t S, int64_t H, int64_t D, float scale, int32_t param_bits,
                                   void* out, void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * sq_attn_decode_kv4_split_noalloc -- sq_attn_decode_kv4_split for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid it): the same kernels, with the partial states in the library's own scratch, a
 * file-scope device array of 8 MiB per GPU, held from its first use until the process
 * ends.  The call allocates nothing and frees nothing.
 * The scratch is shared by every call on the same GPU and keeps the last call's contents
 * (no part of it needs clearing: a call writes every state it reads).  Calls that overlap
 * on one GPU race: order them (same stream, or synchronised).
 * Arguments, layouts and errors as sq_attn_decode_kv4_split without the workspace;
 * SQ_ERR_SHAPE when the split needs more than the 8 MiB (sq_attn_decode_workspace gives
 * the bytes; on MI355X no valid shape needs more than about 4.3 MiB).
 */
sq_status sq_attn_decode_kv4_split_noalloc(const void* q_rot, const uint8_t* k_q, const void* k_alpha,
                                           const void* k_beta, const uint8_t* v_q, const void* v_alpha,
                                           const void* v_beta, int64_t B, int64_t S, int64_t H, int64_t D,
                                           float scale, int32_t param_bits, void* out, void* stream);

/*
 * The paged cache.  A serving program's K/V cache is a pool of pages of `page` tokens, handed to
 * sequences as they grow, with Hkv key/value heads that Hq >= Hkv query heads share (Hq % Hkv == 0;
 * query head h uses key/value head h / (Hq / Hkv)).  Arguments common to the four calls below:
 *
 *   k_q, v_q   device uint8 [pages, Hkv, page, D*bits/8], 16-byte aligned: 4-bit codes packed as
 *              everywhere, or 8-bit codes
 *   params     device [pages, Hkv, page, 4], 16-byte (param_bits 16: 8-byte) aligned: k_alpha, k_beta,
 *              v_alpha, v_beta of each token and head, fp32 or fp16 as in sq_qk_had_kvquant_ex
 *   pages, page, Hkv   1 <= pages < 2^31; page a power of two, 16 <= page <= 2^20; 1 <= Hkv <= 2^16;
 *              pages * page * Hkv <= 2^40
 *   bits, param_bits   4 or 8; 32 or 16 (others: SQ_ERR_UNSUPPORTED)
 *   block_table device int32 [B, ld_table], 4-byte aligned: entry i < max_blocks of row b is the page
 *              that holds the positions i*page .. i*page + page - 1 of sequence b
 *              (1 <= max_blocks <= ld_table).  An entry outside [0, pages), and a position past the
 *              table, has no page: nothing is written there, it reads as zeros, and attention leaves
 *              it out.  Pages may be shared by sequences that only read them.
 *   lens       device int32 [B]: tokens of each sequence in the cache, the ones of this call included
 *   cu         device int32 [B + 1], ascending: the rows cu[b] .. cu[b+1] - 1 of a packed call belong
 *              to sequence b and are its LAST ones: row t has position lens[b] - cu[b+1] + t.  A row
 *              that belongs to no sequence (before cu[0], from cu[B] on), or whose position is
 *              negative, is left alone: none of its outputs is written.
 *   D          128 (others: SQ_ERR_UNSUPPORTED)
 *   ld*        elements from one token's heads to the next one's, >= heads * D and < 2^24, a multiple
 *              of 8: a tensor may be a slice of a fused projection's output
 * lens, cu and the table stay on the device, so that a captured graph can be replayed as sequences
 * grow.  No value in them makes a call read or write outside the tensors.
 */

/*
 * sq_rope_frequencies -- host helper: the angle per position of each pair of dims,
 * f_i = theta^(-2 i / rotary_dim), i < rotary_dim / 2, in out_host[rotary_dim / 2] (HOST memory).
 *   rotary_dim 16 .. 128, a multiple of 16
 *   theta      base, finite and > 0 (a longer base is given here directly), not so small that an f_i
 *              overflows
 *   scaling    0: none; 1: positions interpolated, f_i / factor; 2: by parts: with r = original_len
 *              f_i / (2 pi) turns within the original context, f_i is kept where r >= high, divided
 *              by factor where r <= low, and between the two mixed linearly in r
 *   factor     >= 1, finite (scaling 1, 2);  low < high, original_len > 0, finite (scaling 2)
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED (other scalings).
 */
sq_status sq_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, double low, double high,
                              double original_len, double* out_host);

/*
 * sq_rope_kv_write -- rotary positions and R3 (Sec. 3.1) on the queries and keys of new tokens, per
 * head, and the quantized write of their keys and values into the pages (eq. 1, one group per
 * token and head):
 *     (u, w) -> (u c - w s, w c + u s),  c = magnitude cos(p f_i),  s = magnitude sin(p f_i)
 * for the pair i of the first rotary_dim dims at position p, then y = x S_128 / sqrt(128).
 *   q          device fp16 [T, ldq]: Hq heads of D;  k, v  device fp16 [T, ldk], [T, ldv]: Hkv heads
 *              of D; 16-byte aligned, BEFORE the rotary positions
 *   T          >= 0 rows (0 is a no-op), < 2^31;  1 <= Hq <= 2^16
 *   cu         may be NULL: row t is the one new token of sequence t (T == B)
 *   freq       device fp64 [rotary_dim / 2], radians per position, 8-byte aligned (sq_rope_frequencies
 *              gives them); NULL iff rotary_dim == 0 (no positions: R3 and the write alone)
 *   rotary_dim 0 .. 128, a multiple of 16: the leading dims that turn
 *   interleaved  0: pair i is (i, i + rotary_dim / 2); 1: (2 i, 2 i + 1)
 *   magnitude  finite factor of the turned dims (1 unless a long-context scaling asks for another)
 *   k_clip, v_clip   clipping ratios in (0, 1] as in sq_qk_had_kvquant_ex
 *   q_rot      device fp16 [T, Hq, D] contiguous, 16-byte aligned
 *   k_rot      optional device fp16 [T, Hkv, D] contiguous: the turned keys before quantization
 *              (what a prompt's own attention reads); NULL to skip
 * Angles, and keys up to their one rounding to fp32, are computed in 64 bits: positions of any size
 * keep their angle, and the codes are eq. 1's 32-bit steps on that fp32 key.  Two rows of one call
 * must not meet in one slot (a page in two sequences at a position both write): such a slot holds
 * bytes of either.
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_rope_kv_write(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           int64_t T, int64_t Hq, int64_t D, const int32_t* cu, const int32_t* lens, int64_t B,
                           const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                           uint8_t* k_q, uint8_t* v_q, void* params, int64_t pages, int64_t page, int64_t Hkv,
                           int32_t bits, int32_t param_bits,
                           const double* freq, int32_t rotary_dim, int32_t interleaved, float magnitude,
                           float k_clip, float v_clip, void* q_rot, void* k_rot, void* stream);

/*
 * sq_kv_read -- keys and values of the sequences' last tokens out of the pages: alpha c + beta of
 * eq. 1, rounded to fp16, in packed rows, as sq_attn_prompt reads them.
 *   T          >= 0 rows (0 is a no-op), < 2^31
 *   plain_basis  0: keys as stored, in R3's basis (for rotated queries); 1: turned back
 *   k, v       device fp16 [T, ldk], [T, ldv]: Hkv heads of D, 16-byte aligned; the spans of the two,
 *              gaps between rows included, must not overlap
 * Errors as sq_rope_kv_write.
 */
sq_status sq_kv_read(const int32_t* cu, const int32_t* lens, int64_t B, int64_t T,
                     const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                     const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages, int64_t page, int64_t Hkv,
                     int64_t D, int32_t bits, int32_t param_bits, int32_t plain_basis,
                     void* k, int64_t ldk, void* v, int64_t ldv, void* stream);

/*
 * sq_attn_paged -- attention of one query per sequence and head over its pages, the step that
 * follows sq_rope_kv_write for generated tokens:
 *     out[b,h,:] = fp16( sum_t softmax_t(scale * q[b,h,:] . K_t) V_t ),  t < min(lens[b], max_len),
 * K_t and V_t of key/value head h / (Hq / Hkv).  A sequence without tokens (or without pages) gets
 * zeros, whatever its query holds; with tokens, a query that is not finite gives NaN.  The parameters
 * v_alpha of these tokens must be 2^-60 or more (the library writes no others from fp16 values with a
 * v_clip of 2^-28 or more), or 0 with value codes of 0 (a slot of a zeroed cache that was never
 * written): a token's weight and v_alpha (1 for 0) go into one fp16 factor.  A token whose softmax
 * weight times v_alpha is below 2^-26 of the sequence's largest such product counts with less than
 * that factor's 11 bits, below 2^-38 not at all (2^-14 and 2^-25 where the base-2 scores pass 2^22).
 *   q          device fp16 [B, ldq]: Hq heads of D, 16-byte aligned (q_rot of the write)
 *   B          >= 0 (0 is a no-op), B * Hq < 2^24
 *   max_len    1 <= max_len < 2^30, at least the longest length: it fixes the split of the sequence and
 *              with it the workspace and the order of additions
 *   scale      finite score scale, at most 2^40 in size, e.g. 1/sqrt(128)
 *   out        device fp16 [B, ldo]: Hq heads of D, 16-byte aligned
 *   workspace  device memory, 16-byte aligned, at least the bytes sq_attn_paged_workspace gives (NULL
 *              allowed when that is 0); scratch, must not overlap any argument; calls that share
 *              one must be ordered
 * The result does not depend on the run.  Errors as sq_rope_kv_write; SQ_ERR_SHAPE for a workspace
 * too small.
 */
sq_status sq_attn_paged(const void* q, int64_t ldq, const int32_t* lens, int64_t B,
                        const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                        const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages, int64_t page, int64_t Hkv,
                        int64_t Hq, int64_t D, int32_t bits, int32_t param_bits, int64_t max_len, float scale,
                        void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream);

/* Device bytes of sq_attn_paged's workspace on the CURRENT device.  Errors: SQ_ERR_NULL, SQ_ERR_SHAPE,
 * SQ_ERR_UNSUPPORTED, SQ_ERR_HIP. */
sq_status sq_attn_paged_workspace(int64_t B, int64_t max_len, int64_t Hq, int64_t Hkv, int64_t D, uint64_t* bytes);

/*
 * sq_attn_prompt -- attention of packed sequences in fp16 on the matrix cores: the rows
 * cu_q[b] .. cu_q[b+1] - 1 of q over the rows cu_k[b] .. cu_k[b+1] - 1 of k and v.  With n queries
 * and m keys, query i (from 0) sees the keys t < m (causal 0) or t <= m - n + i (causal 1): the
 * queries are the last n tokens, so a chunk of a prompt comes with the keys of what went before.
 * A query that sees no key gets zeros.  Values and keys that a query does not see have no part in
 * its result, NaN and infinities among them; of what it sees, a NaN score, one of +inf, or none above
 * -inf makes its result NaN, and a value that is not finite makes its dim infinite or NaN.  Softmax
 * weights go into the second product in fp16: a key whose weight is below 2^-21 of its row's largest
 * counts with less than fp16's 11 bits, below 2^-32 not at all (2^-14 and 2^-25 where the base-2 scores
 * pass 2^22, at which fp32 has steps of 1/2).
 *   q          device fp16 [Tq, ldq]: Hq heads of D;  k, v  device fp16 [Tk, ldk], [Tk, ldv]: Hkv heads
 *              of D; 16-byte aligned
 *   cu_q, cu_k device int32 [B + 1], ascending, within [0, Tq] and [0, Tk] (entries beyond are taken as
 *              the end).  Rows of q outside the sequences are left as they were in out.
 *   Tq, Tk     >= 0, < 2^31 (Tq == 0 or B == 0 is a no-op; with Tk == 0 k and v may be NULL)
 *   Hq, Hkv    1 <= Hkv <= Hq <= 2^16, Hq % Hkv == 0; Tq * Hq + 256 * B * Hkv < 2^31
 *   scale      positive finite score scale, at most 2^40
 *   out        device fp16 [Tq, ldo]: Hq heads of D, 16-byte aligned
 *   workspace  as in sq_attn_paged, sized by sq_attn_prompt_workspace (0 where there are rows enough
 *              to fill the device)
 * The result does not depend on the run.  Errors as sq_attn_paged.
 */
sq_status sq_attn_prompt(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                         const int32_t* cu_q, const int32_t* cu_k, int64_t B, int64_t Tq, int64_t Tk,
                         int64_t Hq, int64_t Hkv, int64_t D, float scale, int32_t causal, void* out, int64_t ldo,
                         void* workspace, uint64_t workspace_bytes, void* stream);

/* Device bytes of sq_attn_prompt's workspace on the CURRENT device.  Errors: SQ_ERR_NULL, SQ_ERR_SHAPE,
 * SQ_ERR_UNSUPPORTED, SQ_ERR_HIP. */
sq_status sq_attn_prompt_workspace(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, uint64_t* bytes);

/*
 * Drafted tokens, windows and the pages of a step.
 *
 * A draft is a token that the model has yet to check.  A sequence's drafts of a step are its last n
 * tokens in the cache, rows cu[b] .. cu[b+1] - 1 of the packed calls (n = cu[b+1] - cu[b]), and form a
 * tree: draft i continues its parent, a draft before it, or the text.  Its place in the cache is
 * base + i, base = lens[b] - n; its position in the text is base + depth, depth being the number of
 * its ancestors among the drafts.
 *
 * window > 0 lets a token at position p see the keys at positions t > p - window, itself the last, and
 * besides them the first `sinks` ones, t < sinks; window == 0: all keys before it (sinks counts for
 * nothing then).  0 <= window, sinks < 2^30.
 */

/*
 * sq_tree_mask -- the drafts that each draft sees, and its depth, from the drafts' parents.
 *   parents    device int32 [T]: index of the parent among the sequence's drafts; a value outside
 *              [0, i) at draft i (e.g. -1) makes it a root, which continues the text
 *   cu         device int32 [B + 1], ascending: the sequences' rows; rows of no sequence are left alone
 *   lens       device int32 [B]: tokens in the cache, the drafts included; read, and required, only with
 *              window > 0 and sinks > 0
 *   T, B       >= 0 (0 is a no-op), < 2^31
 *   window, sinks  as above: an ancestor `window` or more steps up is left out, unless its position is
 *              below sinks (none is with sinks 0)
 *   mask       device int32 [T, ld_mask], the first `words` words of a row written: bit j % 32 of word
 *              j / 32 of draft i is 1 where j is i or an ancestor that i sees.  Drafts from 32 * words on
 *              have no bits.
 *   words, ld_mask  1 <= words <= 2^9, words <= ld_mask < 2^24
 *   depth      device int32 [T]
 * A sequence's drafts from 2^14 on get depth 0 and no bits.
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_ALIGN (4 bytes each), SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_tree_mask(const int32_t* parents, const int32_t* cu, const int32_t* lens, int64_t B, int64_t T,
                       int32_t window, int32_t sinks, int32_t* mask, int64_t ld_mask, int64_t words, int32_t* depth,
                       void* stream);

/*
 * sq_rope_kv_write_ex -- sq_rope_kv_write with the rows' positions apart from their places in the cache
 * (sq_rope_kv_write is this call with depth = NULL):
 *   depth      device int32 [T] or NULL: row t of sequence b turns by the position lens[b] - n + depth[t],
 *              n = cu[b+1] - cu[b] (1 without cu), and is written to its place as ever.  The
 *              position of a row that is written is taken as it is, negative ones included.
 * Every other argument, layout and error as sq_rope_kv_write; depth is an input for the overlap check.
 */
sq_status sq_rope_kv_write_ex(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                              int64_t T, int64_t Hq, int64_t D, const int32_t* cu, const int32_t* lens, int64_t B,
                              const int32_t* depth,
                              const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                              uint8_t* k_q, uint8_t* v_q, void* params, int64_t pages, int64_t page, int64_t Hkv,
                              int32_t bits, int32_t param_bits,
                              const double* freq, int32_t rotary_dim, int32_t interleaved, float magnitude,
                              float k_clip, float v_clip, void* q_rot, void* k_rot, void* stream);

/*
 * sq_attn_tree -- attention of a sequence's last n tokens over its pages: drafts, or the tokens of a
 * prompt's chunk, written by sq_rope_kv_write(_ex) before:
 *     out[t,h,:] = fp16( sum_j softmax_j(scale * q[t,h,:] . K_j) V_j ),
 * over the tokens j < min(lens[b], max_len) that row t sees.  Row t = cu[b] + i sees
 *   with mask     the tokens before the drafts, j < base, as far as the window at position base + depth[t]
 *                 lets it, and of the drafts exactly those whose bit is set
 *   without       the tokens j <= base + i, as far as the window at base + i lets it
 * A row that sees no token with a page gets zeros; one with a token that it sees and a query that is
 * not finite gives NaN.  What a row does not see has no part in its result, NaN and infinities among
 * the parameters included; of what it sees, a v_beta that is not finite makes it infinite or NaN.
 * Precision and the range of v_alpha as in sq_attn_paged, row by row: whatever the other rows' queries.
 *   q          device fp16 [T, ldq]: Hq rotated heads of D, 16-byte aligned
 *   cu         device int32 [B + 1], ascending, within [0, T] (values beyond are taken as the end).  Rows
 *              of no sequence, and rows with base + i < 0, are left as they were in out.
 *   mask       device int32 [T, ld_mask] or NULL, as sq_tree_mask writes it (any bits are fine: a row need
 *              not see itself); drafts from 32 * words on are seen by none
 *   words, ld_mask  1 <= words <= 2^16, words <= ld_mask < 2^24 (ignored without mask)
 *   depth      device int32 [T] or NULL (depth i in row i; must be NULL without mask); read with window > 0
 *              alone, and taken as 0 below 0 and as 2^30 above
 *   T          >= 0, T * Hq + B * Hq < 2^24 (T == 0 or B == 0 is a no-op)
 *   max_len    1 <= max_len < 2^30, at least the longest length: with T, B and the window it fixes the
 *              split of the sequence, the workspace and the order of additions
 *   out        device fp16 [T, ldo]: Hq heads of D, 16-byte aligned
 *   workspace  as in sq_attn_paged, sized by sq_attn_tree_workspace for the same sizes
 * Every other argument as in sq_attn_paged.  The result does not depend on the run.  Errors as
 * sq_attn_paged.
 */
sq_status sq_attn_tree(const void* q, int64_t ldq, const int32_t* cu, const int32_t* lens, int64_t B, int64_t T,
                       const int32_t* mask, int64_t ld_mask, int64_t words, const int32_t* depth,
                       int32_t window, int32_t sinks,
                       const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                       const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages, int64_t page, int64_t Hkv,
                       int64_t Hq, int64_t D, int32_t bits, int32_t param_bits, int64_t max_len, float scale,
                       void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream);

/* Device bytes of sq_attn_tree's workspace on the CURRENT device.  Errors: SQ_ERR_NULL, SQ_ERR_SHAPE,
 * SQ_ERR_UNSUPPORTED, SQ_ERR_HIP. */
sq_status sq_attn_tree_workspace(int64_t B, int64_t T, int64_t max_len, int32_t window, int32_t sinks, int64_t Hq, int64_t Hkv,
                                 int64_t D, uint64_t* bytes);

/*
 * sq_attn_paged_window -- sq_attn_paged of a token that sees the last `window` tokens of its sequence and
 * the first `sinks` ones (window 0: all of them).  Pages that lie wholly between the two may have gone
 * back to the pool (sq_paged_release): they are not read.  Token, range of v_alpha, zeros and NaN as in
 * sq_attn_tree.
 *   window, sinks  as above
 *   B          >= 0 (0 is a no-op), 2 * B * Hq < 2^24
 *   workspace  sized by sq_attn_paged_window_workspace for the same sizes
 * Every other argument and error as sq_attn_paged.
 */
sq_status sq_attn_paged_window(const void* q, int64_t ldq, const int32_t* lens, int64_t B, int32_t window, int32_t sinks,
                               const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                               const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages, int64_t page,
                               int64_t Hkv, int64_t Hq, int64_t D, int32_t bits, int32_t param_bits, int64_t max_len,
                               float scale, void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream);

/* Device bytes of sq_attn_paged_window's workspace on the CURRENT device.  Errors as sq_attn_tree_workspace. */
sq_status sq_attn_paged_window_workspace(int64_t B, int64_t max_len, int32_t window, int32_t sinks, int64_t Hq, int64_t Hkv,
                                         int64_t D, uint64_t* bytes);

/*
 * sq_attn_prompt_window -- the causal attention of sq_attn_prompt in which query i of a sequence of n
 * queries and m keys, at position p = m - n + i, sees the keys p - window < t <= p and t < sinks, t <= p
 * (window 0: all up to p).  Keys outside every window of a sequence are not read.
 *   window, sinks  as above
 *   workspace  sized by sq_attn_prompt_window_workspace for the same sizes
 * Every other argument and error as sq_attn_prompt with causal = 1.
 */
sq_status sq_attn_prompt_window(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                const int32_t* cu_q, const int32_t* cu_k, int64_t B, int64_t Tq, int64_t Tk,
                                int64_t Hq, int64_t Hkv, int64_t D, float scale, int32_t window, int32_t sinks,
                                void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream);

/* Device bytes of sq_attn_prompt_window's workspace on the CURRENT device.  Errors as sq_attn_prompt_workspace. */
sq_status sq_attn_prompt_window_workspace(int64_t B, int64_t Tq, int64_t Tk, int32_t window, int32_t sinks, int64_t Hq,
                                          int64_t Hkv, int64_t D, uint64_t* bytes);

/*
 * The pages of the pool on the device, so that a captured step can hand them out.  Common to the two calls:
 *   pool       device int32 [pages]: its first count[0] entries are the free pages; a page is taken from
 *              the end and goes back there
 *   count      device int32 [1], in and out; taken as within [0, pages]
 *   held       device int32 [B], in and out: the blocks of each sequence that have a page, the first
 *              held[b] columns of its row of the table; taken as within [0, max_blocks]
 *   block_table, ld_table, max_blocks, page   as in the paged calls; in and out
 *   B          >= 0 (0 is a no-op of sq_paged_release), <= 2^20;  max_blocks < 2^24, pages < 2^31
 * Calls that share a pool, a table or held must be ordered.  All is decided by the values on the device;
 * none of them makes a call read or write outside the tensors.
 */

/*
 * sq_paged_release -- pages go back to the pool: of sequence b the held blocks whose positions all lie in
 * first[b] .. end[b] - 1.  end may lie past the last token: at or past the end of the last held block,
 * held[b] becomes the first block that went (what ended a sequence, first = 0, or took back its drafts,
 * first = tokens kept); below it held[b] stays (what a window has left behind of the tokens so far: end =
 * tokens - window, which is below it; first = sinks in a sequence's first call, then the largest `end` so far
 * rounded down to a whole block, but sinks at least).  Their entries become -1; one that is not a page of the
 * pool goes nowhere.  The pages join the pool by sequence, then block.  A page that two sequences share must
 * be released by one of them alone.  Every block of the range is looked at, those that have gone before too:
 * with first = sinks in every call a window would look at the whole text behind it each time, for the same
 * result.
 *   first, end device int32 [B]; first below 0 counts as 0
 * Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_paged_release(const int32_t* first, const int32_t* end, int32_t* held, int64_t B,
                           int32_t* block_table, int64_t ld_table, int64_t max_blocks, int64_t page,
                           int32_t* pool, int32_t* count, int64_t pages, void* stream);

/*
 * sq_paged_grow -- pages, lengths and rows of a step's new tokens: sequence b has have[b] tokens in the cache
 * and gets add[b] (below 0: 0).  Its blocks up to the last new token that have no page yet get pages of the
 * pool, by sequence, then block; then
 *   lens       device int32 [B]: have + add, what the calls of the step take
 *   cu         device int32 [B + 1]: the rows of each sequence's new tokens, cu[0] = 0
 *   pos        device int32 [T]: the position have[b] + i of row cu[b] + i; -1 in rows from cu[B] on
 *   slots      device int64 [T]: where the row's token lies, page * (tokens of a page) + place, the index
 *              among a head's tokens of the pool; -1 in rows from cu[B] on, and where the table's entry is
 *              not a page of the pool
 *   missing    device int32 [2]: the pages that the pool, or columns that the table, lacks for this, and the
 *              rows that T lacks; (0, 0) when all is well.  Otherwise nothing is handed out: table, held and
 *              count stay, lens is have, cu is 0, pos and slots are -1, so that the calls of the step have no
 *              rows, and the step can be tried again when pages have come back.
 *   T          >= 0 rows of pos and slots (0: both may be NULL), < 2^31
 * Sums beyond 2^31 - 1 count as that many.  Errors as sq_paged_release.
 */
sq_status sq_paged_grow(const int32_t* have, const int32_t* add, int32_t* held, int64_t B, int64_t T,
                        int32_t* block_table, int64_t ld_table, int64_t max_blocks, int64_t page,
                        int32_t* pool, int32_t* count, int64_t pages,
                        int32_t* lens, int32_t* cu, int32_t* pos, int64_t* slots, int32_t* missing, void* stream);

/*
 * sq_kv_keep -- after the check of a step's drafts: those of the accepted path become the sequence's next
 * tokens.  Draft path[b][i], i < kept[b], moves to the place base + i, codes and parameters as they are, in
 * all heads; the sequence then has lens_out[b] = base + kept[b] tokens.  (Draft path[b][i] of a tree has
 * depth i, so its key is turned for the position that it moves to.)
 *   path       device int32 [B, ld_path], the first max_kept entries of a row: indexes of drafts on the way
 *              down a tree (parents before children, so that entry i is i or more)
 *   kept       device int32 [B], taken as within [0, min(n, max_kept)]
 *   max_kept   1 <= max_kept <= ld_path < 2^24
 *   cu, lens   as in sq_attn_tree, before the move; base and places below 0 have no token
 *   lens_out   device int32 [B], at least 0; not lens itself, which is read while it is written
 * An entry outside [i, n), or whose place or whose draft has no page, moves nothing: the place keeps what it
 * held.  Errors: SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP.
 */
sq_status sq_kv_keep(const int32_t* cu, const int32_t* lens, int64_t B, const int32_t* path, int64_t ld_path, int64_t max_kept,
                     const int32_t* kept, const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                     uint8_t* k_q, uint8_t* v_q, void* params, int64_t pages, int64_t page, int64_t Hkv,
                     int64_t D, int32_t bits, int32_t param_bits, int32_t* lens_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SQ_H_ */
