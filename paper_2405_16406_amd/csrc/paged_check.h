// Argument checks shared by the host sources of the paged cache's entry points.
#pragma once

#include <cmath>

#include "api_check.h"

namespace sq::api {

constexpr int64_t kMost32 = (int64_t{1} << 31) - 1;

inline uint64_t rows_bytes(int64_t rows, int64_t ld, int64_t heads) {
  return rows ? (static_cast<uint64_t>(rows - 1) * ld + heads * 128) * 2 : 0;
}

inline sq_status check_ld(int64_t ld, int64_t heads, const char* name) {
  if (ld < heads * 128 || ld >= (int64_t{1} << 24))
    return fail(SQ_ERR_SHAPE, "%s=%lld outside [%lld, 2^24)", name, (long long)ld, (long long)(heads * 128));
  if (ld % 8 != 0) return fail(SQ_ERR_ALIGN, "%s=%lld is not a multiple of 8", name, (long long)ld);
  return SQ_OK;
}

inline sq_status check_heads(int64_t Hq, int64_t Hkv, int64_t D) {
  if (D != 128) return fail(SQ_ERR_UNSUPPORTED, "D=%lld: only head_dim 128 is implemented", (long long)D);
  if (Hkv < 1 || Hq < Hkv || Hq > (1 << 16) || Hq % Hkv != 0)
    return fail(SQ_ERR_SHAPE, "Hq=%lld, Hkv=%lld: need 1 <= Hkv <= Hq <= 2^16 and Hq %% Hkv == 0", (long long)Hq, (long long)Hkv);
  return SQ_OK;
}

// The kernels multiply by log2(e) scale, the paged one by 2^24 more: kMostScale keeps both finite.
constexpr float kMostScale = 1099511627776.0f;  // 2^40
inline sq_status check_scale(float scale, bool positive) {
  if (!(std::fabs(scale) <= kMostScale)) return fail(SQ_ERR_SHAPE, "scale must be finite and at most 2^40 in size");
  // (the prompt kernel takes the maximum of the unscaled scores)
  if (positive && !(scale > 0.0f)) return fail(SQ_ERR_SHAPE, "scale must be positive");
  return SQ_OK;
}

constexpr int64_t kMostWindow = int64_t{1} << 30;

inline sq_status check_window(int32_t window, int32_t sinks) {
  if (window < 0 || sinks < 0 || window >= kMostWindow || sinks >= kMostWindow)
    return fail(SQ_ERR_SHAPE, "window=%d and sinks=%d must lie in [0, 2^30)", window, sinks);
  return SQ_OK;
}

// The cache arguments; fills c and the bytes of its codes (each) and parameters.
inline sq_status check_cache(const int32_t* table, int64_t ldt, int64_t cols, const uint8_t* kq, const uint8_t* vq, const void* params,
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

inline uint64_t table_bytes(int64_t B, int64_t ldt, int64_t cols) { return B ? (static_cast<uint64_t>(B - 1) * ldt + cols) * 4 : 0; }

inline sq_status check_workspace(const void* workspace, uint64_t bytes, uint64_t need) {
  if (bytes < need || (need > 0 && !workspace))
    return fail(SQ_ERR_SHAPE, "workspace of %llu bytes, %llu needed", (unsigned long long)bytes, (unsigned long long)need);
  return SQ_OK;
}

inline float log2_scale(float scale) { return static_cast<float>(static_cast<double>(scale) * 1.4426950408889634); }

}  // namespace sq::api
