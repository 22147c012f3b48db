// The host-compilable parts of the windowed prompt attention, for tests/test_prompt_window_host.py.
#include "paged.h"
#include "paged_plan.h"

extern "C" {

// half, splits and tiles of a part, as sq_attn_prompt_window plans them.
void window_plan(int64_t B, int64_t Tq, int64_t Tk, int32_t window, int32_t sinks, int32_t hq, int32_t hkv, int cus, int32_t* out) {
  const sq::PromptPlan p = sq::prompt_plan(B, Tq, sq::window_keys(B, Tk, window, sinks), hq, hkv, cus);
  out[0] = p.half;
  out[1] = p.splits;
  out[2] = p.per;
}

// head, start and tokens of the run of a tile of rows at positions low .. last.
void tile_run(int32_t low, int32_t last, int32_t window, int32_t sinks, int32_t* out) {
  const sq::TokenRun r = sq::token_run(low, last + 1, window, sinks);
  out[0] = r.head;
  out[1] = r.start;
  out[2] = r.tokens;
}

int32_t window_part(int32_t tiles, int32_t splits, int32_t per) { return sq::prompt_part(tiles, splits, per); }
}
