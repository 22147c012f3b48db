// How the write of the paged cache and the attention over it and over prompts are split over
// workgroups: sizes alone (no HIP), so that the host compiles and checks it too.
#pragma once

#include <cstdint>

#include "paged.h"

namespace sq {

// The write.  A wave's worth of vectors of n tokens (a task): 16 queries, 8 keys or 16 values each.
struct RopeTasks {
  int q, k, v;
  SQ_HOST_DEVICE int all() const { return q + k + v; }
};
SQ_HOST_DEVICE RopeTasks rope_tasks(int n, int hq, int hkv) {
  return {(n * hq + 15) / 16, (n * hkv + 7) / 8, (n * hkv + 15) / 16};
}
constexpr int kRopeWaves = 8;   // of a workgroup at most
constexpr int kRopeTokens = 8;  // tokens of a workgroup at most

// Many rows: workgroups of four waves with up to four tasks each, the next one's vectors on their way
// while one is worked on, as long as 1024 of them (four a CU) are left.  A CU holds four only of the
// forms with up to 128 registers (8 bits, or fp16 parameters, with rotary_dim 0 or 128 in halves), else
// three.  Few rows (a decode step): a wave for each task, for the shortest way through.  Measured, us
// with the read back: 17034 rows of 32 + 32 heads 237 (four waves of four tasks), 241 (eight of four),
// 284 (sixteen of one).
struct RopePlan {
  int tokens, waves;  // of a workgroup
};
inline RopePlan rope_plan(int64_t T, int hq, int hkv) {
  constexpr int kMany = 1024, kLoop = 4;
  int tokens = 1;
  while (2 * tokens <= kRopeTokens && T >= 2 * tokens * kMany && rope_tasks(2 * tokens, hq, hkv).all() <= kLoop * kLoop) tokens *= 2;
  const int most = T >= kMany ? kLoop : kRopeWaves, tasks = rope_tasks(tokens, hq, hkv).all();
  return {tokens, tasks < most ? tasks : most};
}

constexpr int kPagedWaves = 4;    // of a decode workgroup, each on its own
constexpr int kPagedBlock = 64;   // tokens of a wave's step

// Decode: tokens of a chunk (whole steps of a workgroup) and chunks of the longest sequence.
//   One sequence: two workgroups for each of `cus` compute units, one round of equal ones (131071
//   tokens of 8 heads, us with the join: chunks of 2048 tokens 34, 1536 37, 8192 54).
//   Several: their lengths differ as a rule, so four times as many, the sequences' short last chunks
//   among them filling up at the end (64 sequences of 512 .. 8192 tokens, 8 heads: 2048 53, 8192 77;
//   equal lengths lose by it, 64 of 2432: 43, uncut 38).  Chunks of one step for each wave only where
//   there is nothing better to do for the compute units (16 sequences, 8 heads: 512 15, 256 16).
// The lengths lie on the device, so the plan goes by the longest.
inline void paged_split(int64_t B, int64_t max_len, int32_t hq, int32_t hkv, int cus, int32_t& chunks, int32_t& chunk_tokens) {
  constexpr int64_t unit = kPagedWaves * kPagedBlock;
  const int64_t groups = B * hkv * ((hq / hkv + 15) / 16);
  const int64_t tokens = groups * max_len;  // < 2^54
  const int64_t want = static_cast<int64_t>(cus) * (B > 1 ? 8 : 2);
  int64_t chunk = (tokens + want - 1) / want;
  const int64_t least = tokens / unit > 4 * static_cast<int64_t>(cus) ? 2 * unit : unit;
  if (chunk < least) chunk = least;
  chunk = (chunk + unit - 1) / unit * unit;
  if (chunk > max_len) chunk = (max_len + unit - 1) / unit * unit;
  chunk_tokens = static_cast<int32_t>(chunk < unit ? unit : chunk);
  chunks = static_cast<int32_t>((max_len + chunk_tokens - 1) / chunk_tokens);
  if (chunks < 1) chunks = 1;
}

// Several rows of a sequence over its pages: workgroups of `waves` waves for 16 * rb (row, query head) pairs,
// `tiles` of them at most, and the tokens that they see in `chunks` pieces of chunk_tokens.
//   rb: a column of 16 rows, or two that share the expanded codes.  Two need whole columns, and work enough that half
//   the workgroups still fill the compute units (64 drafts behind 131008 tokens, 32 heads on 8, us: one column 315, two
//   219; 8 behind 131008 with 8 bits 73 and 65; 16 behind 2048 12.8 and 13.5).
//   chunks: as in decode above for up to 16 rows; more work longer on a token, and of several sequences half as
//   many pieces do (16 sequences of 4096 tokens, 64 rows, 8 heads: 1024 tokens 26.6, 512 33.6, 2048 30.4).
//   Windows shorter than the sequences make their runs as good as equal: one round, as of one sequence (64
//   of 512 .. 8192 tokens in windows of 2048, 8 heads: uncut 33.9, 768 tokens 44.4).
//   waves: short runs of few workgroups stay uncut, with eight waves each, which spares the join's launch (16
//   drafts behind L tokens, 4 bits, eager calls and on the device alone, us: L = 512 12.9 and 8.8, cut 16.8 and
//   10.9; 1024 12.9 and 11.0, cut 17.0 and 11.0; 2048 15.4 and 15.3, cut 17.0 and 13.1; 4096 with 8 bits 28, cut 16).
constexpr int kWideRun = 5 * kPagedWaves * kPagedBlock;
struct TreePlan {
  int32_t rb, waves, tiles, chunks, chunk_tokens;
};
inline TreePlan tree_plan(int64_t B, int64_t T, bool single, int64_t max_len, int32_t window, int32_t sinks, int32_t hq, int32_t hkv,
                          int cus) {
  constexpr int64_t unit = kPagedWaves * kPagedBlock;
  const int64_t group = hq / hkv, rows = T * group, some = B > 0 ? B : 1;
  TreePlan p{};
  // tokens of the longest run: the window of the first row, the rows behind it, and what whole blocks add
  int64_t run = max_len;
  if (window > 0) {
    const int64_t most = static_cast<int64_t>(sinks) + window + (single ? 1 : T) + 2 * kPagedBlock;
    if (run > most) run = most;
  }
  const int64_t each = (rows + some - 1) / some;  // rows of an average sequence
  const bool two = each > 16 && some * ((each + 31) / 32) * hkv * ((run + unit - 1) / unit) >= cus;
  p.rb = two ? 2 : 1;
  const int64_t tile = 16 * p.rb;
  p.tiles = static_cast<int32_t>(single ? B * ((group + tile - 1) / tile) : (rows + B * (tile - 1)) / tile);
  const int64_t tokens = some * ((each + 31) / 32) * hkv * run;  // < 2^54
  const bool equal = B == 1 || run < max_len;
  const int64_t want = static_cast<int64_t>(cus) * (equal ? 2 : each > 16 ? 4 : 8);
  int64_t chunk = (tokens + want - 1) / want;
  const int64_t least = tokens / unit > 4 * static_cast<int64_t>(cus) ? 2 * unit : unit;
  if (chunk < least) chunk = least;
  chunk = (chunk + unit - 1) / unit * unit;
  if (chunk > run) chunk = (run + unit - 1) / unit * unit;
  p.waves = kPagedWaves;
  p.chunk_tokens = static_cast<int32_t>(chunk < unit ? unit : chunk);
  if (!two && run > p.chunk_tokens && run <= kWideRun && static_cast<int64_t>(p.tiles) * hkv <= cus) {
    p.waves = 2 * kPagedWaves;
    p.chunk_tokens = static_cast<int32_t>((run + 2 * unit - 1) / (2 * unit) * (2 * unit));
  }
  p.chunks = static_cast<int32_t>((run + p.chunk_tokens - 1) / p.chunk_tokens);
  if (p.chunks < 1) p.chunks = 1;
  return p;
}

constexpr int kPromptRows = 256;  // (token, query head) rows of a prompt workgroup
constexpr int kPromptTile = 64;   // keys of its step

// Prompts.  half: workgroups of half the rows, whose two groups of waves share the keys.  splits > 1:
// the keys go out in parts of `per` tiles (more where a sequence would have over `splits` of them).
//   Workgroups of 256 rows for more of them than compute units: they move the fewest bytes through
//   the caches (prompt of 4096 tokens of 32 heads: 143 us, halves 158; 8192: 517, 560).
//   Up to one a compute unit, the longest of a causal prompt decides: halves (2048 tokens 50 us,
//   whole 57; 1024: 24, 33; 512: 16, 23).
//   Few rows over many keys: parts, a unit each, where by the estimate below they are through
//   sooner, partial states included (37 and 4 tokens over 16000 and 6000 keys of 8 heads 34 us).
struct PromptPlan {
  int32_t half, splits, per;
};

inline PromptPlan prompt_plan(int64_t B, int64_t Tq, int64_t Tk, int32_t hq, int32_t hkv, int cus) {
  if (B < 1 || Tq < 1 || Tk < 1) return {0, 1, 0};
  const int64_t tiles = (Tq * (hq / hkv) + kPromptRows - 1) / kPromptRows;
  const int64_t groups = (tiles > B ? tiles : B) * hkv;
  if (groups > cus) return {0, 1, 0};
  const int64_t keys = (Tk + kPromptTile - 1) / kPromptTile;
  // A part of each sequence, row tile and head is half empty on average; four tiles or more.
  const int64_t work = keys * hkv * ((tiles + B - 1) / B), units = cus - groups / 2;
  int64_t per = (work + units - 1) / units;
  if (per < 4) per = 4;
  int64_t splits = (keys + per - 1) / per;
  // partial states of 132 floats a row and part: at most 2^18 of them
  const int64_t rows = Tq * hq, most = (int64_t{1} << 18) / rows;
  if (splits > most) splits = most;
  if (splits < 2) return {1, 1, 0};
  // In steps of a tile (2 us): halves take every second tile of an average sequence, in one or two
  // rounds; parts their own, three more steps, and the states' way to memory and back (3 TB/s).
  const int64_t halves = (keys / B + 1) / 2 * ((2 * groups + cus - 1) / cus);
  const int64_t parts = per + 3 + rows * splits * 1056 / 6000000;
  if (halves <= parts) return {1, 1, 0};
  return {0, static_cast<int32_t>(splits), static_cast<int32_t>(per)};
}

// What a window leaves of Tk keys: the run of a tile of rows holds at most its sinks and window, its rows and what
// whole blocks of 64 add.
inline int64_t window_keys(int64_t B, int64_t Tk, int32_t window, int32_t sinks) {
  if (window <= 0) return Tk;
  const int64_t most = (B > 1 ? B : 1) * (static_cast<int64_t>(sinks) + window + kPromptRows + 2 * kPromptTile);
  return most < Tk ? most : Tk;
}

// Tiles of a part of a sequence (or of a tile of its rows) with `tiles` of them.
SQ_HOST_DEVICE int32_t prompt_part(int32_t tiles, int32_t splits, int32_t per) {
  const int32_t least = (tiles + splits - 1) / splits;
  return per > least ? per : least;
}

}  // namespace sq
