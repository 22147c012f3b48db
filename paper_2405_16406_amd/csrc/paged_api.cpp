// Host side of the paged-cache entry points of include/sq.h: argument validation and launches.
// Every check runs before anything is enqueued.
#include <algorithm>
#include <cmath>

#include "api_check.h"
#include "paged_plan.h"

namespace {

using namespace sq::api;

constexpr int64_t kMost32 = (int64_t{1} << 31) - 1;

uint64_t rows_bytes(int64_t rows, int64_t ld, int64_t heads) {
  return rows ? (static_cast<uint64_t>(rows - 1) * ld + heads * 128) * 2 : 0;
}

sq_status check_ld(int64_t ld, int64_t heads, const char* name) {
  if (ld < heads * 128 || ld >= (int64_t{1} << 24))
    return fail(SQ_ERR_SHAPE, "%s=%lld outside [%lld, 2^24)", name, (long long)ld, (long long)(heads * 128));
  if (ld % 8 != 0) return fail(SQ_ERR_ALIGN, "%s=%lld is not a multiple of 8", name, (long long)ld);
  return SQ_OK;
}

sq_status check_heads(int64_t Hq, int64_t Hkv, int64_t D) {
  if (D != 128) return fail(SQ_ERR_UNSUPPORTED, "D=%lld: only head_dim 128 is implemented", (long long)D);
  if (Hkv < 1 || Hq < Hkv || Hq > (1 << 16) || Hq % Hkv != 0)
    return fail(SQ_ERR_SHAPE, "Hq=%lld, Hkv=%lld: need 1 <= Hkv <= Hq <= 2^16 and Hq %% Hkv == 0", (long long)Hq, (long long)Hkv);
  return SQ_OK;
}

// The kernels multiply by log2(e) scale, the paged one by 2^24 more: kMostScale keeps both finite.
constexpr float kMostScale = 1099511627776.0f;  // 2^40
sq_status check_scale(float scale, bool positive) {
  if (!(std::fabs(scale) <= kMostScale)) return fail(SQ_ERR_SHAPE, "scale must be finite and at most 2^40 in size");
  // (the prompt kernel takes the maximum of the unscaled scores)
  if (positive && !(scale > 0.0f)) return fail(SQ_ERR_SHAPE, "scale must be positive");
  return SQ_OK;
}

// The cache arguments; fills c and the bytes of its codes (each) and parameters.
sq_status check_cache(const int32_t* table, int64_t ldt, int64_t cols, const uint8_t* kq, const uint8_t* vq, const void* params,
                      int64_t pages, int64_t page, int64_t Hkv, int64_t D, int32_t bits, int32_t param_bits, const int32_t* lens,
                      int64_t B, sq::PagedCache& c, uint64_t& code_bytes, uint64_t& param_bytes) {
  if (!table || !kq || !vq || !params || !lens) return fail(SQ_ERR_NULL, "block_table, lens, k_q, v_q and params are required");
  if (D != 128) return fail(SQ_ERR_UNSUPPORTED, "D=%lld: only head_dim 128 is implemented", (long long)D);
  if (bits != 4 && bits != 8) return fail(SQ_ERR_UNSUPPORTED, "bits=%d: 4- and 8-bit caches are implemented", bits);
  if (param_bits != 32 && param_bits != 16)
    return fail(SQ_ERR_UNSUPPORTED, "param_bits=%d: fp32 (32) and fp16 (16) group parameters are implemented", param_bits);
  if (B < 0 || B > kMost32) return fail(SQ_ERR_SHAPE, "B=%lld out of range", (long long)B);
  if (!is_pow2(page) || page < 16 || page > (1 << 20))
    return fail(SQ_ERR_SHAPE, "page=%lld is not a power of two in [16, 2^20]", (long long)page);
  if (Hkv < 1 || Hkv > (1 << 16)) return fail(SQ_ERR_SHAPE, "Hkv=%lld outside [1, 2^16]", (long long)Hkv);
  if (pages < 1 || pages > kMost32 || pages > (int64_t{1} << 40) / (page * Hkv))
    return fail(SQ_ERR_SHAPE, "pages=%lld out of range", (long long)pages);
  if (cols < 1 || cols > kMost32 || ldt < cols || ldt > (int64_t{1} << 40))
    return fail(SQ_ERR_SHAPE, "need 1 <= max_blocks=%lld <= ld_table=%lld", (long long)cols, (long long)ldt);
  const uintptr_t pa = param_bits / 2;  // 16 or 8 bytes a record
  if (!aligned(kq, 16) || !aligned(vq, 16) || !aligned(params, pa) || !aligned(table, 4) || !aligned(lens, 4))
    return fail(SQ_ERR_ALIGN, "k_q and v_q need 16-byte, params %d-byte, lens and block_table 4-byte alignment", static_cast<int>(pa));
  const uint64_t slots = static_cast<uint64_t>(pages) * page * Hkv;
  code_bytes = slots * 16 * bits;
  param_bytes = slots * pa;
  c = sq::PagedCache{};
  c.kq = const_cast<uint8_t*>(kq);
  c.vq = const_cast<uint8_t*>(vq);
  c.params = const_cast<void*>(params);
  c.table = table;
  c.ldt = ldt;
  c.cols = static_cast<int32_t>(cols);
  c.pages = static_cast<int32_t>(pages);
  while ((int64_t{1} << c.shift) < page) ++c.shift;
  c.heads = static_cast<int32_t>(Hkv);
  return SQ_OK;
}

uint64_t table_bytes(int64_t B, int64_t ldt, int64_t cols) { return B ? (static_cast<uint64_t>(B - 1) * ldt + cols) * 4 : 0; }

// The split of sq_attn_paged on the current device, and the workspace bytes it needs.
sq_status paged_split_here(int64_t B, int64_t max_len, int64_t Hq, int64_t Hkv, int32_t& chunks, int32_t& tokens, uint64_t& bytes) {
  int cus = 0;
  const hipError_t e = sq::device_cus(&cus);
  if (e != hipSuccess) return hip_status(e, "compute-unit count of the current device");
  sq::paged_split(B, max_len, static_cast<int32_t>(Hq), static_cast<int32_t>(Hkv), cus, chunks, tokens);
  bytes = chunks > 1 ? static_cast<uint64_t>(B) * Hq * chunks * (sq::kAttnPart * 4) : 0;
  return SQ_OK;
}

sq_status check_paged_sizes(int64_t B, int64_t max_len, int64_t Hq, int64_t Hkv, int64_t D) {
  const sq_status s = check_heads(Hq, Hkv, D);
  if (s != SQ_OK) return s;
  if (B < 0 || B >= (int64_t{1} << 24) / Hq) return fail(SQ_ERR_SHAPE, "B=%lld: need B * Hq < 2^24", (long long)B);
  if (max_len < 1 || max_len >= (int64_t{1} << 30)) return fail(SQ_ERR_SHAPE, "max_len=%lld outside [1, 2^30)", (long long)max_len);
  return SQ_OK;
}

sq_status prompt_plan_here(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, sq::PromptPlan& plan, uint64_t& bytes) {
  int cus = 0;
  const hipError_t e = sq::device_cus(&cus);
  if (e != hipSuccess) return hip_status(e, "compute-unit count of the current device");
  plan = sq::prompt_plan(B, Tq, Tk, static_cast<int32_t>(Hq), static_cast<int32_t>(Hkv), cus);
  bytes = plan.splits > 1 ? static_cast<uint64_t>(Tq) * Hq * plan.splits * (sq::kAttnPart * 4) : 0;
  return SQ_OK;
}

sq_status check_prompt_sizes(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D) {
  const sq_status s = check_heads(Hq, Hkv, D);
  if (s != SQ_OK) return s;
  if (B < 0 || Tq < 0 || Tk < 0 || B > kMost32 || Tq > kMost32 || Tk > kMost32)
    return fail(SQ_ERR_SHAPE, "B=%lld, Tq=%lld or Tk=%lld out of range", (long long)B, (long long)Tq, (long long)Tk);
  if (Tq * Hq + 256 * B * Hkv > kMost32)
    return fail(SQ_ERR_SHAPE, "Tq * Hq + 256 * B * Hkv = %lld beyond 2^31", (long long)(Tq * Hq + 256 * B * Hkv));
  return SQ_OK;
}

sq_status check_workspace(const void* workspace, uint64_t bytes, uint64_t need) {
  if (bytes < need || (need > 0 && !workspace))
    return fail(SQ_ERR_SHAPE, "workspace of %llu bytes, %llu needed", (unsigned long long)bytes, (unsigned long long)need);
  return SQ_OK;
}

float log2_scale(float scale) { return static_cast<float>(static_cast<double>(scale) * 1.4426950408889634); }

}  // namespace

extern "C" {

sq_status sq_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, double low, double high,
                              double original_len, double* out_host) {
  if (!out_host) return fail(SQ_ERR_NULL, "out_host is NULL");
  if (rotary_dim < 16 || rotary_dim > 128 || rotary_dim % 16 != 0)
    return fail(SQ_ERR_SHAPE, "rotary_dim=%d is not a multiple of 16 in [16, 128]", rotary_dim);
  if (!(theta > 0.0) || !std::isfinite(theta)) return fail(SQ_ERR_SHAPE, "theta must be finite and positive");
  if (scaling < 0 || scaling > 2) return fail(SQ_ERR_UNSUPPORTED, "scaling=%d: 0, 1 and 2 are implemented", scaling);
  if (scaling > 0 && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(SQ_ERR_SHAPE, "factor must be finite and at least 1");
  if (scaling == 2 && (!(low < high) || !std::isfinite(low) || !std::isfinite(high) || !(original_len > 0.0) || !std::isfinite(original_len)))
    return fail(SQ_ERR_SHAPE, "need finite low < high and original_len > 0");
  double out[64];
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / rotary_dim);
    if (scaling == 1) f /= factor;
    if (scaling == 2) {
      const double turns = original_len * f / 6.283185307179586477;
      double kept = (turns - low) / (high - low);
      kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
      f = f * kept + f / factor * (1.0 - kept);
    }
    if (!std::isfinite(f)) return fail(SQ_ERR_SHAPE, "theta=%g: the frequency of pair %d is not finite", theta, i);
    out[i] = f;
  }
  std::copy(out, out + rotary_dim / 2, out_host);
  return ok();
}

sq_status sq_rope_kv_write(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           int64_t T, int64_t Hq, int64_t D, const int32_t* cu, const int32_t* lens, int64_t B,
                           const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                           uint8_t* k_q, uint8_t* v_q, void* params, int64_t pages, int64_t page, int64_t Hkv,
                           int32_t bits, int32_t param_bits,
                           const double* freq, int32_t rotary_dim, int32_t interleaved, float magnitude,
                           float k_clip, float v_clip, void* q_rot, void* k_rot, void* stream) {
  TimingScope timing_scope;
  if (!q || !k || !v || !q_rot) return fail(SQ_ERR_NULL, "q, k, v and q_rot are required");
  sq::RopeWriteArgs a{};
  uint64_t codes = 0, pbytes = 0;
  sq_status s = check_cache(block_table, ld_table, max_blocks, k_q, v_q, params, pages, page, Hkv, D, bits, param_bits, lens, B,
                            a.cache, codes, pbytes);
  if (s != SQ_OK || (s = check_heads(Hq, Hkv, D)) != SQ_OK) return s;
  if (T < 0 || T > kMost32) return fail(SQ_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if (!cu && T != B) return fail(SQ_ERR_SHAPE, "without cu every sequence has one row: T=%lld, B=%lld", (long long)T, (long long)B);
  if ((s = check_ld(ldq, Hq, "ldq")) != SQ_OK || (s = check_ld(ldk, Hkv, "ldk")) != SQ_OK || (s = check_ld(ldv, Hkv, "ldv")) != SQ_OK)
    return s;
  if (rotary_dim < 0 || rotary_dim > 128 || rotary_dim % 16 != 0)
    return fail(SQ_ERR_SHAPE, "rotary_dim=%d is not a multiple of 16 in [0, 128]", rotary_dim);
  if ((rotary_dim == 0) != (freq == nullptr))
    return fail(rotary_dim == 0 ? SQ_ERR_SHAPE : SQ_ERR_NULL, "freq must be NULL iff rotary_dim == 0 (%d)", rotary_dim);
  if (interleaved != 0 && interleaved != 1) return fail(SQ_ERR_UNSUPPORTED, "interleaved=%d: 0 and 1 are implemented", interleaved);
  if (!(std::fabs(magnitude) < 3.0e38f)) return fail(SQ_ERR_SHAPE, "magnitude must be finite");
  if ((s = check_clip(k_clip, "k_clip")) != SQ_OK || (s = check_clip(v_clip, "v_clip")) != SQ_OK) return s;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_rot, 16) || !aligned(k_rot, 16) || !aligned(cu, 4) ||
      !aligned(freq, 8))
    return fail(SQ_ERR_ALIGN, "q, k, v, q_rot and k_rot need 16-byte, freq 8-byte and cu 4-byte alignment");
  s = check_alias({{q, rows_bytes(T, ldq, Hq), "q"}, {k, rows_bytes(T, ldk, Hkv), "k"}, {v, rows_bytes(T, ldv, Hkv), "v"},
                   {cu, static_cast<uint64_t>(B + 1) * 4, "cu"}, {lens, static_cast<uint64_t>(B) * 4, "lens"},
                   {block_table, table_bytes(B, ld_table, max_blocks), "block_table"},
                   {freq, static_cast<uint64_t>(rotary_dim) * 4, "freq"}},
                  {{q_rot, static_cast<uint64_t>(T) * Hq * 256, "q_rot"}, {k_rot, static_cast<uint64_t>(T) * Hkv * 256, "k_rot"},
                   {k_q, codes, "k_q"}, {v_q, codes, "v_q"}, {params, pbytes, "params"}});
  if (s != SQ_OK) return s;
  if (T == 0 || B == 0) return ok();
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldv = ldv;
  a.T = T;
  a.hq = static_cast<int32_t>(Hq);
  a.cu = cu;
  a.lens = lens;
  a.B = B;
  a.freq = freq;
  a.rotary = rotary_dim;
  a.interleaved = interleaved;
  a.magnitude = magnitude;
  a.k_clip = k_clip;
  a.v_clip = v_clip;
  a.bits = bits;
  a.param16 = param_bits == 16;
  a.q_rot = static_cast<uint16_t*>(q_rot);
  a.k_rot = static_cast<uint16_t*>(k_rot);
  return hip_status(sq::launch_rope_kv_write(a, static_cast<hipStream_t>(stream)), "rope_kv_write launch");
}

sq_status sq_kv_read(const int32_t* cu, const int32_t* lens, int64_t B, int64_t T,
                     const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                     const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages, int64_t page, int64_t Hkv,
                     int64_t D, int32_t bits, int32_t param_bits, int32_t plain_basis,
                     void* k, int64_t ldk, void* v, int64_t ldv, void* stream) {
  TimingScope timing_scope;
  if (!cu || !k || !v) return fail(SQ_ERR_NULL, "cu, k and v are required");
  sq::KvReadArgs a{};
  uint64_t codes = 0, pbytes = 0;
  sq_status s = check_cache(block_table, ld_table, max_blocks, k_q, v_q, params, pages, page, Hkv, D, bits, param_bits, lens, B,
                            a.cache, codes, pbytes);
  if (s != SQ_OK) return s;
  if (T < 0 || T > kMost32) return fail(SQ_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if ((s = check_ld(ldk, Hkv, "ldk")) != SQ_OK || (s = check_ld(ldv, Hkv, "ldv")) != SQ_OK) return s;
  if (plain_basis != 0 && plain_basis != 1) return fail(SQ_ERR_UNSUPPORTED, "plain_basis=%d: 0 and 1 are implemented", plain_basis);
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cu, 4)) return fail(SQ_ERR_ALIGN, "k and v need 16-byte, cu 4-byte alignment");
  s = check_alias({{cu, static_cast<uint64_t>(B + 1) * 4, "cu"}, {lens, static_cast<uint64_t>(B) * 4, "lens"},
                   {block_table, table_bytes(B, ld_table, max_blocks), "block_table"}, {k_q, codes, "k_q"}, {v_q, codes, "v_q"},
                   {params, pbytes, "params"}},
                  {{k, rows_bytes(T, ldk, Hkv), "k"}, {v, rows_bytes(T, ldv, Hkv), "v"}});
  if (s != SQ_OK) return s;
  if (T == 0 || B == 0) return ok();
  a.cu = cu;
  a.lens = lens;
  a.B = B;
  a.T = T;
  a.bits = bits;
  a.param16 = param_bits == 16;
  a.plain_basis = plain_basis;
  a.k = static_cast<uint16_t*>(k);
  a.v = static_cast<uint16_t*>(v);
  a.ldk = ldk;
  a.ldv = ldv;
  return hip_status(sq::launch_kv_read(a, static_cast<hipStream_t>(stream)), "kv_read launch");
}

sq_status sq_attn_paged_workspace(int64_t B, int64_t max_len, int64_t Hq, int64_t Hkv, int64_t D, uint64_t* bytes) {
  if (!bytes) return fail(SQ_ERR_NULL, "bytes is required");
  sq_status s = check_paged_sizes(B, max_len, Hq, Hkv, D);
  if (s != SQ_OK) return s;
  int32_t chunks = 1, tokens = 0;
  uint64_t need = 0;
  if ((s = paged_split_here(B, max_len, Hq, Hkv, chunks, tokens, need)) != SQ_OK) return s;
  *bytes = need;
  return ok();
}

sq_status sq_attn_paged(const void* q, int64_t ldq, const int32_t* lens, int64_t B,
                        const int32_t* block_table, int64_t ld_table, int64_t max_blocks,
                        const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages, int64_t page, int64_t Hkv,
                        int64_t Hq, int64_t D, int32_t bits, int32_t param_bits, int64_t max_len, float scale,
                        void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream) {
  TimingScope timing_scope;
  if (!q || !out) return fail(SQ_ERR_NULL, "q and out are required");
  sq::PagedAttnArgs a{};
  uint64_t codes = 0, pbytes = 0;
  sq_status s = check_cache(block_table, ld_table, max_blocks, k_q, v_q, params, pages, page, Hkv, D, bits, param_bits, lens, B,
                            a.cache, codes, pbytes);
  if (s != SQ_OK || (s = check_paged_sizes(B, max_len, Hq, Hkv, D)) != SQ_OK || (s = check_ld(ldq, Hq, "ldq")) != SQ_OK ||
      (s = check_ld(ldo, Hq, "ldo")) != SQ_OK || (s = check_scale(scale, false)) != SQ_OK)
    return s;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
    return fail(SQ_ERR_ALIGN, "q, out and the workspace need 16-byte alignment");
  s = check_alias({{q, rows_bytes(B, ldq, Hq), "q"}, {lens, static_cast<uint64_t>(B) * 4, "lens"},
                   {block_table, table_bytes(B, ld_table, max_blocks), "block_table"}, {k_q, codes, "k_q"}, {v_q, codes, "v_q"},
                   {params, pbytes, "params"}},
                  {{out, rows_bytes(B, ldo, Hq), "out"}, {workspace, workspace_bytes, "workspace"}});
  if (s != SQ_OK) return s;
  if (B == 0) return ok();
  uint64_t need = 0;
  if ((s = paged_split_here(B, max_len, Hq, Hkv, a.chunks, a.chunk_tokens, need)) != SQ_OK) return s;
  if ((s = check_workspace(workspace, workspace_bytes, need)) != SQ_OK) return s;
  a.q = static_cast<const uint16_t*>(q);
  a.ldq = ldq;
  a.lens = lens;
  a.B = B;
  a.hq = static_cast<int32_t>(Hq);
  a.group = static_cast<int32_t>(Hq / Hkv);
  a.bits = bits;
  a.param16 = param_bits == 16;
  a.max_len = static_cast<int32_t>(max_len);
  a.scale_log2e = log2_scale(scale);
  a.out = static_cast<uint16_t*>(out);
  a.ldo = ldo;
  a.part = static_cast<float*>(workspace);
  return hip_status(sq::launch_attn_paged(a, static_cast<hipStream_t>(stream)), "attn_paged launch");
}

sq_status sq_attn_prompt_workspace(int64_t B, int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hkv, int64_t D, uint64_t* bytes) {
  if (!bytes) return fail(SQ_ERR_NULL, "bytes is required");
  sq_status s = check_prompt_sizes(B, Tq, Tk, Hq, Hkv, D);
  if (s != SQ_OK) return s;
  sq::PromptPlan plan{};
  uint64_t need = 0;
  if ((s = prompt_plan_here(B, Tq, Tk, Hq, Hkv, plan, need)) != SQ_OK) return s;
  *bytes = need;
  return ok();
}

sq_status sq_attn_prompt(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                         const int32_t* cu_q, const int32_t* cu_k, int64_t B, int64_t Tq, int64_t Tk,
                         int64_t Hq, int64_t Hkv, int64_t D, float scale, int32_t causal, void* out, int64_t ldo,
                         void* workspace, uint64_t workspace_bytes, void* stream) {
  TimingScope timing_scope;
  if (!q || !out || !cu_q || !cu_k || (Tk > 0 && (!k || !v))) return fail(SQ_ERR_NULL, "q, k, v, cu_q, cu_k and out are required");
  sq_status s = check_prompt_sizes(B, Tq, Tk, Hq, Hkv, D);
  if (s != SQ_OK || (s = check_ld(ldq, Hq, "ldq")) != SQ_OK || (s = check_ld(ldk, Hkv, "ldk")) != SQ_OK ||
      (s = check_ld(ldv, Hkv, "ldv")) != SQ_OK || (s = check_ld(ldo, Hq, "ldo")) != SQ_OK || (s = check_scale(scale, true)) != SQ_OK)
    return s;
  if (causal != 0 && causal != 1) return fail(SQ_ERR_UNSUPPORTED, "causal=%d: 0 and 1 are implemented", causal);
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(cu_q, 4) ||
      !aligned(cu_k, 4))
    return fail(SQ_ERR_ALIGN, "q, k, v, out and the workspace need 16-byte, cu_q and cu_k 4-byte alignment");
  s = check_alias({{q, rows_bytes(Tq, ldq, Hq), "q"}, {k, rows_bytes(Tk, ldk, Hkv), "k"}, {v, rows_bytes(Tk, ldv, Hkv), "v"},
                   {cu_q, static_cast<uint64_t>(B + 1) * 4, "cu_q"}, {cu_k, static_cast<uint64_t>(B + 1) * 4, "cu_k"}},
                  {{out, rows_bytes(Tq, ldo, Hq), "out"}, {workspace, workspace_bytes, "workspace"}});
  if (s != SQ_OK) return s;
  if (Tq == 0 || B == 0) return ok();
  sq::PromptArgs a{};
  sq::PromptPlan plan{};
  uint64_t need = 0;
  if ((s = prompt_plan_here(B, Tq, Tk, Hq, Hkv, plan, need)) != SQ_OK) return s;
  a.half = plan.half;
  a.splits = plan.splits;
  a.per = plan.per;
  if ((s = check_workspace(workspace, workspace_bytes, need)) != SQ_OK) return s;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldv = ldv;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.B = B;
  a.Tq = Tq;
  a.Tk = Tk;
  a.hq = static_cast<int32_t>(Hq);
  a.hkv = static_cast<int32_t>(Hkv);
  a.group = static_cast<int32_t>(Hq / Hkv);
  a.scale_log2e = log2_scale(scale);
  a.causal = causal;
  a.out = static_cast<uint16_t*>(out);
  a.ldo = ldo;
  a.part = static_cast<float*>(workspace);
  return hip_status(sq::launch_attn_prompt(a, static_cast<hipStream_t>(stream)), "attn_prompt launch");
}

}  // extern "C"
