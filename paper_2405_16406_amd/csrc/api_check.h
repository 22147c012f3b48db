// Argument checks and error state shared by the host sources of the C ABI (include/sq.h).
#pragma once

#include <cstdint>
#include <initializer_list>
#include <vector>

#include "sq.h"
#include "sq_internal.h"

namespace sq::api {

// Disarms sq_time_next_call's events when the entry point returns, on every path.
struct TimingScope {
  ~TimingScope();
};

// Sets the thread's last error and returns s.
sq_status fail(sq_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears it.
sq_status ok();
sq_status hip_status(hipError_t e, const char* what);

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool is_pow2(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }

struct Range {
  const void* p;
  uint64_t bytes;
  const char* name;
};

inline bool overlap(const Range& a, const Range& b) {
  if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// Outputs must not overlap any input or each other (a list of ranges or a vector of them).
template <typename Ins, typename Outs>
sq_status check_ranges(const Ins& ins, const Outs& outs) {
  for (auto out = outs.begin(); out != outs.end(); ++out) {
    for (const Range& in : ins)
      if (overlap(*out, in)) return fail(SQ_ERR_ALIAS, "output %s overlaps input %s", out->name, in.name);
    for (auto other = out + 1; other != outs.end(); ++other)
      if (overlap(*out, *other)) return fail(SQ_ERR_ALIAS, "output %s overlaps output %s", out->name, other->name);
  }
  return SQ_OK;
}
inline sq_status check_alias(std::initializer_list<Range> ins, std::initializer_list<Range> outs) {
  return check_ranges(ins, outs);
}
inline sq_status check_alias(std::initializer_list<Range> ins, const std::vector<Range>& outs) {
  return check_ranges(ins, outs);
}

// A range clipping ratio: finite, 0 < r <= 1.
sq_status check_clip(float r, const char* name);

}  // namespace sq::api
