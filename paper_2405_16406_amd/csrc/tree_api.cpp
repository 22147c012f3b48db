// Host side of the calls around drafted tokens, windows of single tokens and page tables (include/sq.h): argument
// validation and launches.  Every check runs before anything is enqueued.
#include "paged_check.h"
#include "paged_plan.h"

namespace {

using namespace sq::api;

sq_status check_words(int64_t words, int64_t ld_mask) {
  if (words < 1 || words > (1 << 16) || ld_mask < words || ld_mask >= (int64_t{1} << 24))
    return fail(SQ_ERR_SHAPE, "need 1 <= words=%lld <= 2^16 and words <= ld_mask=%lld < 2^24", (long long)words, (long long)ld_mask);
  return SQ_OK;
}

uint64_t mask_bytes(int64_t T, int64_t ld_mask, int64_t words) { return T ? (static_cast<uint64_t>(T - 1) * ld_mask + words) * 4 : 0; }

sq_status check_tree_sizes(int64_t B, int64_t T, int64_t max_len, int32_t window, int32_t sinks, int64_t Hq, int64_t Hkv, int64_t D) {
  sq_status s = check_heads(Hq, Hkv, D);
  if (s != SQ_OK || (s = check_window(window, sinks)) != SQ_OK) return s;
  if (B < 0 || T < 0 || B > kMost32 || T > kMost32 || T + B >= ((int64_t{1} << 24) + Hq - 1) / Hq)
    return fail(SQ_ERR_SHAPE, "T=%lld, B=%lld: need (T + B) * Hq < 2^24", (long long)T, (long long)B);
  if (max_len < 1 || max_len >= (int64_t{1} << 30)) return fail(SQ_ERR_SHAPE, "max_len=%lld outside [1, 2^30)", (long long)max_len);
  return SQ_OK;
}

// The plan on the current device, and the workspace bytes it needs.
sq_status tree_plan_here(int64_t B, int64_t T, bool single, int64_t max_len, int32_t window, int32_t sinks, int64_t Hq, int64_t Hkv,
                         sq::TreePlan& plan, uint64_t& bytes) {
  int cus = 0;
  const hipError_t e = sq::device_cus(&cus);
  if (e != hipSuccess) return hip_status(e, "compute-unit count of the current device");
  plan = sq::tree_plan(B, T, single, max_len, window, sinks, static_cast<int32_t>(Hq), static_cast<int32_t>(Hkv), cus);
  bytes = plan.chunks > 1 ? static_cast<uint64_t>(T) * Hq * plan.chunks * (sq::kAttnPart * 4) : 0;
  return SQ_OK;
}

// sq_attn_tree, and with cu NULL (one row a sequence) sq_attn_paged_window.
sq_status attn_tree(const void* q, int64_t ldq, const int32_t* cu, bool single, const int32_t* lens, int64_t B, int64_t T,
                    const int32_t* mask, int64_t ld_mask, int64_t words, const int32_t* depth, int32_t window, int32_t sinks,
                    const int32_t* block_table, int64_t ld_table, int64_t max_blocks, const uint8_t* k_q, const uint8_t* v_q,
                    const void* params, int64_t pages, int64_t page, int64_t Hkv, int64_t Hq, int64_t D, int32_t bits, int32_t param_bits,
                    int64_t max_len, float scale, void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!q || !out || (!single && !cu)) return fail(SQ_ERR_NULL, "q, cu and out are required");
  sq::TreeArgs a{};
  uint64_t codes = 0, pbytes = 0;
  sq_status s = check_cache(block_table, ld_table, max_blocks, k_q, v_q, params, pages, page, Hkv, D, bits, param_bits, lens, B,
                            a.cache, codes, pbytes);
  if (s != SQ_OK || (s = check_tree_sizes(B, T, max_len, window, sinks, Hq, Hkv, D)) != SQ_OK ||
      (s = check_ld(ldq, Hq, "ldq")) != SQ_OK || (s = check_ld(ldo, Hq, "ldo")) != SQ_OK || (s = check_scale(scale, false)) != SQ_OK)
    return s;
  if (mask && (s = check_words(words, ld_mask)) != SQ_OK) return s;
  if (depth && !mask) return fail(SQ_ERR_SHAPE, "depth without mask: a chain's depths are its rows");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(cu, 4) || !aligned(mask, 4) || !aligned(depth, 4))
    return fail(SQ_ERR_ALIGN, "q, out and the workspace need 16-byte, cu, mask and depth 4-byte alignment");
  s = check_alias({{q, rows_bytes(T, ldq, Hq), "q"}, {cu, static_cast<uint64_t>(B + 1) * 4, "cu"},
                   {lens, static_cast<uint64_t>(B) * 4, "lens"}, {mask, mask_bytes(T, ld_mask, words), "mask"},
                   {depth, static_cast<uint64_t>(T) * 4, "depth"}, {block_table, table_bytes(B, ld_table, max_blocks), "block_table"},
                   {k_q, codes, "k_q"}, {v_q, codes, "v_q"}, {params, pbytes, "params"}},
                  {{out, rows_bytes(T, ldo, Hq), "out"}, {workspace, workspace_bytes, "workspace"}});
  if (s != SQ_OK) return s;
  if (T == 0 || B == 0) return ok();
  uint64_t need = 0;
  if ((s = tree_plan_here(B, T, single, max_len, window, sinks, Hq, Hkv, a.plan, need)) != SQ_OK) return s;
  if ((s = check_workspace(workspace, workspace_bytes, need)) != SQ_OK) return s;
  a.q = static_cast<const uint16_t*>(q);
  a.ldq = ldq;
  a.cu = cu;
  a.lens = lens;
  a.B = B;
  a.T = T;
  a.mask = mask;
  a.ldm = ld_mask;
  a.words = static_cast<int32_t>(words);
  a.depth = depth;
  a.window = window;
  a.sinks = window > 0 ? sinks : 0;
  a.hq = static_cast<int32_t>(Hq);
  a.group = static_cast<int32_t>(Hq / Hkv);
  a.bits = bits;
  a.param16 = param_bits == 16;
  a.max_len = static_cast<int32_t>(max_len);
  a.scale_log2e = log2_scale(scale);
  a.out = static_cast<uint16_t*>(out);
  a.ldo = ldo;
  a.part = static_cast<float*>(workspace);
  return hip_status(sq::launch_attn_tree(a, static_cast<hipStream_t>(stream)), "attn_tree launch");
}

// The arguments that the two calls on page tables share.
sq_status check_pool(const int32_t* held, int64_t B, int32_t* table, int64_t ldt, int64_t cols, int64_t page, int32_t* pool, int32_t* count,
                     int64_t pages, sq::PoolArgs& p) {
  if (!held || !table || !pool || !count) return fail(SQ_ERR_NULL, "held, block_table, pool and count are required");
  if (B < 0 || B > (1 << 20)) return fail(SQ_ERR_SHAPE, "B=%lld outside [0, 2^20]", (long long)B);
  if (!is_pow2(page) || page < 16 || page > (1 << 20))
    return fail(SQ_ERR_SHAPE, "page=%lld is not a power of two in [16, 2^20]", (long long)page);
  if (pages < 1 || pages > kMost32) return fail(SQ_ERR_SHAPE, "pages=%lld out of range", (long long)pages);
  if (cols < 1 || cols >= (1 << 24) || ldt < cols || ldt > (int64_t{1} << 40))
    return fail(SQ_ERR_SHAPE, "need 1 <= max_blocks=%lld < 2^24 and max_blocks <= ld_table=%lld", (long long)cols, (long long)ldt);
  if (!aligned(held, 4) || !aligned(table, 4) || !aligned(pool, 4) || !aligned(count, 4))
    return fail(SQ_ERR_ALIGN, "held, block_table, pool and count need 4-byte alignment");
  p = sq::PoolArgs{};
  p.held = const_cast<int32_t*>(held);
  p.B = B;
  p.table = table;
  p.ldt = ldt;
  p.cols = static_cast<int32_t>(cols);
  while ((int64_t{1} << p.shift) < page) ++p.shift;
  p.pool = pool;
  p.count = count;
  p.pages = static_cast<int32_t>(pages);
  return SQ_OK;
}

}  // namespace

extern "C" {

sq_status sq_tree_mask(const int32_t* parents, const int32_t* cu, const int32_t* lens, int64_t B, int64_t T, int32_t window, int32_t sinks,
                       int32_t* mask, int64_t ld_mask, int64_t words, int32_t* depth, void* stream) {
  TimingScope timing_scope;
  if (!parents || !cu || !mask || !depth) return fail(SQ_ERR_NULL, "parents, cu, mask and depth are required");
  sq_status s = check_window(window, sinks);
  if (s != SQ_OK || (s = check_words(words, ld_mask)) != SQ_OK) return s;
  if (words > sq::kMaskDrafts / 32) return fail(SQ_ERR_SHAPE, "words=%lld: a sequence has at most 2^14 drafts", (long long)words);
  const bool first = window > 0 && sinks > 0;
  if (first && !lens) return fail(SQ_ERR_NULL, "lens is required with window and sinks");
  if (B < 0 || T < 0 || B > kMost32 || T > kMost32) return fail(SQ_ERR_SHAPE, "B=%lld or T=%lld out of range", (long long)B, (long long)T);
  if (!aligned(parents, 4) || !aligned(cu, 4) || !aligned(lens, 4) || !aligned(mask, 4) || !aligned(depth, 4))
    return fail(SQ_ERR_ALIGN, "parents, cu, lens, mask and depth need 4-byte alignment");
  const uint64_t rows = static_cast<uint64_t>(T) * 4;
  s = check_alias({{parents, rows, "parents"}, {cu, static_cast<uint64_t>(B + 1) * 4, "cu"},
                   {first ? lens : nullptr, static_cast<uint64_t>(B) * 4, "lens"}},
                  {{mask, mask_bytes(T, ld_mask, words), "mask"}, {depth, rows, "depth"}});
  if (s != SQ_OK) return s;
  if (B == 0 || T == 0) return ok();
  sq::TreeMaskArgs a{};
  a.parents = parents;
  a.cu = cu;
  a.lens = first ? lens : nullptr;
  a.B = B;
  a.T = T;
  a.window = window;
  a.sinks = sinks;
  a.mask = mask;
  a.ldm = ld_mask;
  a.words = static_cast<int32_t>(words);
  a.depth = depth;
  return hip_status(sq::launch_tree_mask(a, static_cast<hipStream_t>(stream)), "tree_mask launch");
}

sq_status sq_attn_tree_workspace(int64_t B, int64_t T, int64_t max_len, int32_t window, int32_t sinks, int64_t Hq, int64_t Hkv, int64_t D,
                                 uint64_t* bytes) {
  if (!bytes) return fail(SQ_ERR_NULL, "bytes is required");
  sq_status s = check_tree_sizes(B, T, max_len, window, sinks, Hq, Hkv, D);
  if (s != SQ_OK) return s;
  sq::TreePlan plan{};
  uint64_t need = 0;
  if ((s = tree_plan_here(B, T, false, max_len, window, sinks, Hq, Hkv, plan, need)) != SQ_OK) return s;
  *bytes = need;
  return ok();
}

sq_status sq_attn_tree(const void* q, int64_t ldq, const int32_t* cu, const int32_t* lens, int64_t B, int64_t T, const int32_t* mask,
                       int64_t ld_mask, int64_t words, const int32_t* depth, int32_t window, int32_t sinks, const int32_t* block_table,
                       int64_t ld_table, int64_t max_blocks, const uint8_t* k_q, const uint8_t* v_q, const void* params, int64_t pages,
                       int64_t page, int64_t Hkv, int64_t Hq, int64_t D, int32_t bits, int32_t param_bits, int64_t max_len, float scale,
                       void* out, int64_t ldo, void* workspace, uint64_t workspace_bytes, void* stream) {
  TimingScope timing_scope;
  return attn_tree(q, ldq, cu, false, lens, B, T, mask, ld_mask, words, depth, window, sinks, block_table, ld_table, max_blocks, k_q, v_q,
                   params, pages, page, Hkv, Hq, D, bits, param_bits, max_len, scale, out, ldo, workspace, workspace_bytes, stream);
}

sq_status sq_attn_paged_window_workspace(int64_t B, int64_t max_len, int32_t window, int32_t sinks, int64_t Hq, int64_t Hkv, int64_t D,
                                         uint64_t* bytes) {
  if (!bytes) return fail(SQ_ERR_NULL, "bytes is required");
  sq_status s = check_tree_sizes(B, B, max_len, window, sinks, Hq, Hkv, D);
  if (s != SQ_OK) return s;
  sq::TreePlan plan{};
  uint64_t need = 0;
  if ((s = tree_plan_here(B, B, true, max_len, window, sinks, Hq, Hkv, plan, need)) != SQ_OK) return s;
  *bytes = need;
  return ok();
}

sq_status sq_attn_paged_window(const void* q, int64_t ldq, const int32_t* lens, int64_t B, int32_t window, int32_t sinks,
                               const int32_t* block_table, int64_t ld_table, int64_t max_blocks, const uint8_t* k_q, const uint8_t* v_q,
                               const void* params, int64_t pages, int64_t page, int64_t Hkv, int64_t Hq, int64_t D, int32_t bits,
                               int32_t param_bits, int64_t max_len, float scale, void* out, int64_t ldo, void* workspace,
                               uint64_t workspace_bytes, void* stream) {
  TimingScope timing_scope;
  return attn_tree(q, ldq, nullptr, true, lens, B, B, nullptr, 0, 0, nullptr, window, sinks, block_table, ld_table, max_blocks, k_q, v_q,
                   params, pages, page, Hkv, Hq, D, bits, param_bits, max_len, scale, out, ldo, workspace, workspace_bytes, stream);
}

sq_status sq_paged_release(const int32_t* first, const int32_t* end, int32_t* held, int64_t B, int32_t* block_table, int64_t ld_table,
                           int64_t max_blocks, int64_t page, int32_t* pool, int32_t* count, int64_t pages, void* stream) {
  TimingScope timing_scope;
  if (!first || !end) return fail(SQ_ERR_NULL, "first and end are required");
  sq::PoolArgs p{};
  sq_status s = check_pool(held, B, block_table, ld_table, max_blocks, page, pool, count, pages, p);
  if (s != SQ_OK) return s;
  if (!aligned(first, 4) || !aligned(end, 4)) return fail(SQ_ERR_ALIGN, "first and end need 4-byte alignment");
  const uint64_t each = static_cast<uint64_t>(B) * 4;
  s = check_alias({{first, each, "first"}, {end, each, "end"}},
                  {{held, each, "held"}, {block_table, table_bytes(B, ld_table, max_blocks), "block_table"},
                   {pool, static_cast<uint64_t>(pages) * 4, "pool"}, {count, 4, "count"}});
  if (s != SQ_OK) return s;
  if (B == 0) return ok();
  return hip_status(sq::launch_paged_release(p, first, end, static_cast<hipStream_t>(stream)), "paged_release launch");
}

sq_status sq_paged_grow(const int32_t* have, const int32_t* add, int32_t* held, int64_t B, int64_t T, int32_t* block_table, int64_t ld_table,
                        int64_t max_blocks, int64_t page, int32_t* pool, int32_t* count, int64_t pages, int32_t* lens, int32_t* cu,
                        int32_t* pos, int64_t* slots, int32_t* missing, void* stream) {
  TimingScope timing_scope;
  if (!have || !add || !lens || !cu || !missing || (T > 0 && (!pos || !slots)))
    return fail(SQ_ERR_NULL, "have, add, lens, cu, pos, slots and missing are required");
  sq::PoolArgs p{};
  sq_status s = check_pool(held, B, block_table, ld_table, max_blocks, page, pool, count, pages, p);
  if (s != SQ_OK) return s;
  if (T < 0 || T > kMost32) return fail(SQ_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if (!aligned(have, 4) || !aligned(add, 4) || !aligned(lens, 4) || !aligned(cu, 4) || !aligned(pos, 4) || !aligned(missing, 4) ||
      !aligned(slots, 8))
    return fail(SQ_ERR_ALIGN, "slots need 8-byte, have, add, lens, cu, pos and missing 4-byte alignment");
  const uint64_t each = static_cast<uint64_t>(B) * 4, rows = static_cast<uint64_t>(T);
  s = check_alias({{have, each, "have"}, {add, each, "add"}},
                  {{held, each, "held"}, {block_table, table_bytes(B, ld_table, max_blocks), "block_table"},
                   {pool, static_cast<uint64_t>(pages) * 4, "pool"}, {count, 4, "count"}, {lens, each, "lens"}, {cu, each + 4, "cu"},
                   {pos, rows * 4, "pos"}, {slots, rows * 8, "slots"}, {missing, 8, "missing"}});
  if (s != SQ_OK) return s;
  sq::GrowArgs g{have, add, T, lens, cu, pos, slots, missing};
  return hip_status(sq::launch_paged_grow(p, g, static_cast<hipStream_t>(stream)), "paged_grow launch");
}

sq_status sq_kv_keep(const int32_t* cu, const int32_t* lens, int64_t B, const int32_t* path, int64_t ld_path, int64_t max_kept,
                     const int32_t* kept, const int32_t* block_table, int64_t ld_table, int64_t max_blocks, uint8_t* k_q, uint8_t* v_q,
                     void* params, int64_t pages, int64_t page, int64_t Hkv, int64_t D, int32_t bits, int32_t param_bits,
                     int32_t* lens_out, void* stream) {
  TimingScope timing_scope;
  if (!cu || !path || !kept || !lens_out) return fail(SQ_ERR_NULL, "cu, path, kept and lens_out are required");
  sq::KeepArgs a{};
  uint64_t codes = 0, pbytes = 0;
  sq_status s = check_cache(block_table, ld_table, max_blocks, k_q, v_q, params, pages, page, Hkv, D, bits, param_bits, lens, B,
                            a.cache, codes, pbytes);
  if (s != SQ_OK) return s;
  if (max_kept < 1 || ld_path < max_kept || ld_path >= (int64_t{1} << 24))
    return fail(SQ_ERR_SHAPE, "need 1 <= max_kept=%lld <= ld_path=%lld < 2^24", (long long)max_kept, (long long)ld_path);
  if (!aligned(cu, 4) || !aligned(path, 4) || !aligned(kept, 4) || !aligned(lens_out, 4))
    return fail(SQ_ERR_ALIGN, "cu, path, kept and lens_out need 4-byte alignment");
  const uint64_t each = static_cast<uint64_t>(B) * 4;
  s = check_alias({{cu, each + 4, "cu"}, {lens, each, "lens"}, {path, table_bytes(B, ld_path, max_kept), "path"}, {kept, each, "kept"},
                   {block_table, table_bytes(B, ld_table, max_blocks), "block_table"}},
                  {{k_q, codes, "k_q"}, {v_q, codes, "v_q"}, {params, pbytes, "params"}, {lens_out, each, "lens_out"}});
  if (s != SQ_OK) return s;
  if (B == 0) return ok();
  a.cu = cu;
  a.lens = lens;
  a.B = B;
  a.path = path;
  a.ldp = ld_path;
  a.most = static_cast<int32_t>(max_kept);
  a.kept = kept;
  a.bits = bits;
  a.param16 = param_bits == 16;
  a.lens_out = lens_out;
  return hip_status(sq::launch_kv_keep(a, static_cast<hipStream_t>(stream)), "kv_keep launch");
}

}  // extern "C"
