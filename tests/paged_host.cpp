// The host-compilable parts of the paged cache, for tests/test_paged_host.py.
#include "paged.h"
#include "paged_plan.h"

extern "C" {

// Slot of row t of a sequence whose rows end before `end` (len tokens in the cache), head h; the
// lookups in the kernels' order, -1 where the row has no place.
int64_t row_slot(int32_t len, int32_t end, int64_t t, const int32_t* table_row, int32_t cols, int32_t pages, int32_t shift,
                 int32_t heads, int32_t h) {
  sq::PagedCache c{};
  c.cols = cols;
  c.pages = pages;
  c.shift = shift;
  c.heads = heads;
  const int64_t pos = sq::row_position(len, end, t);
  const int32_t col = sq::table_column(c, pos);
  if (col < 0) return -1;
  const int32_t page = sq::valid_page(c, table_row[col]);
  return page < 0 ? -1 : sq::token_slot(c, page, h, pos);
}

void paged_split(int64_t B, int64_t max_len, int32_t hq, int32_t hkv, int cus, int32_t* out) {
  sq::paged_split(B, max_len, hq, hkv, cus, out[0], out[1]);
}

void prompt_plan(int64_t B, int64_t Tq, int64_t Tk, int32_t hq, int32_t hkv, int cus, int32_t* out) {
  const sq::PromptPlan p = sq::prompt_plan(B, Tq, Tk, hq, hkv, cus);
  out[0] = p.half;
  out[1] = p.splits;
  out[2] = p.per;
}

void rope_plan(int64_t T, int32_t hq, int32_t hkv, int32_t* out) {
  const sq::RopePlan p = sq::rope_plan(T, hq, hkv);
  out[0] = p.tokens;
  out[1] = p.waves;
}

int32_t prompt_part(int32_t tiles, int32_t splits, int32_t per) { return sq::prompt_part(tiles, splits, per); }
}
