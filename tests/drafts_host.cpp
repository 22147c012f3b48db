// The host-compilable parts of the attention of several rows over the pages, for tests/test_drafts_host.py.
#include "paged.h"
#include "paged_plan.h"

extern "C" {

void token_run(int32_t low, int32_t end, int32_t window, int32_t sinks, int32_t* out) {
  const sq::TokenRun r = sq::token_run(low, end, window, sinks);
  out[0] = r.head;
  out[1] = r.start;
  out[2] = r.tokens;
}

int32_t run_position(int32_t head, int32_t start, int32_t place) { return sq::TokenRun{head, start, 0}.position(place); }

void tree_plan(int64_t B, int64_t T, int32_t single, int64_t max_len, int32_t window, int32_t sinks, int32_t hq, int32_t hkv, int cus,
               int32_t* out) {
  const sq::TreePlan p = sq::tree_plan(B, T, single != 0, max_len, window, sinks, hq, hkv, cus);
  out[0] = p.rb;
  out[1] = p.tiles;
  out[2] = p.chunks;
  out[3] = p.chunk_tokens;
}

int32_t tree_waves(int64_t B, int64_t T, int32_t single, int64_t max_len, int32_t window, int32_t sinks, int32_t hq, int32_t hkv, int cus) {
  return sq::tree_plan(B, T, single != 0, max_len, window, sinks, hq, hkv, cus).waves;
}
}
