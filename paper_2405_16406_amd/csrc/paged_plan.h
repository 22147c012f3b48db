// How the attention over the paged cache and over prompts is split over workgroups: sizes alone
// (no HIP), so that the host compiles and checks it too.
#pragma once

#include <cstdint>

namespace sq {

constexpr int kPagedWaves = 4;    // of a decode workgroup, each on its own
constexpr int kPagedBlock = 64;   // tokens of a wave's step

// Decode: tokens of a chunk (whole steps of a workgroup) and chunks of the longest sequence, for
// about eight workgroups of the longest length on each of `cus` compute units: lengths differ, and
// a chunk that a sequence does not reach ends at once.
inline void paged_split(int64_t B, int64_t max_len, int32_t hq, int32_t hkv, int cus, int32_t& chunks, int32_t& chunk_tokens) {
  constexpr int64_t unit = kPagedWaves * kPagedBlock;
  const int64_t groups = B * hkv * ((hq / hkv + 15) / 16);
  const int64_t want = 8 * static_cast<int64_t>(cus);
  int64_t n = groups > 0 && groups < want ? (want + groups - 1) / groups : 1;
  const int64_t blocks = (max_len + unit - 1) / unit;
  if (n > blocks) n = blocks;
  if (n < 1) n = 1;
  chunk_tokens = static_cast<int32_t>((blocks + n - 1) / n * unit);
  if (chunk_tokens < unit) chunk_tokens = unit;
  chunks = static_cast<int32_t>((max_len + chunk_tokens - 1) / chunk_tokens);
  if (chunks < 1) chunks = 1;
}

constexpr int kPromptRows = 256;  // (token, query head) rows of a prompt workgroup
constexpr int kPromptTile = 64;   // keys of its step

// Prompts: parts that the keys are split into where the rows do not fill the device, eight steps
// or more each on an average sequence.
inline int32_t prompt_splits(int64_t B, int64_t Tq, int64_t Tk, int32_t hq, int32_t hkv, int cus) {
  if (B < 1) return 1;
  const int64_t tiles = (Tq * (hq / hkv) + kPromptRows - 1) / kPromptRows;
  const int64_t groups = (tiles > B ? tiles : B) * hkv;
  if (groups >= cus) return 1;
  int64_t s = cus / groups;
  const int64_t most = Tk / B / (8 * kPromptTile);
  if (s > most) s = most;
  return static_cast<int32_t>(s < 1 ? 1 : s);
}

}  // namespace sq
