// The paged K/V cache: where a row of a packed call belongs and where a token lies in the pool.
// Index arithmetic alone (no HIP), so that the host compiles it too.
//
// Pool: codes of K and of V [pages][heads][page][64 (4 bits) or 128 (8 bits)] bytes and group
// parameters [pages][heads][page][4] (k_alpha, k_beta, v_alpha, v_beta; fp32 or fp16).  The
// tokens of one head are contiguous within a page: a wave that reads 16 tokens of a head reads
// 1 KB of 4-bit codes in whole lines, whatever the number of heads.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define SQ_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define SQ_HOST_DEVICE inline
#endif

namespace sq {

struct PagedCache {
  uint8_t* kq;
  uint8_t* vq;
  void* params;
  const int32_t* table;  // [B, ldt] page of each block of `page` positions
  int64_t ldt;
  int32_t cols;          // valid columns of the table
  int32_t pages;         // pages in the pool
  int32_t shift;         // page = 1 << shift tokens
  int32_t heads;
};

// Position of row t of a packed call in its sequence, whose rows end before row `end` and whose
// cache holds `len` tokens with them.  Negative: the row has no place.
SQ_HOST_DEVICE int64_t row_position(int32_t len, int32_t end, int64_t t) {
  return static_cast<int64_t>(len) - end + t;
}

// Column of the block table that position pos falls into, -1 past the table.
SQ_HOST_DEVICE int32_t table_column(const PagedCache& c, int64_t pos) {
  const int64_t col = pos >> c.shift;
  return pos >= 0 && col < c.cols ? static_cast<int32_t>(col) : -1;
}

// A table entry as a page of the pool, -1 for one that is not.
SQ_HOST_DEVICE int32_t valid_page(const PagedCache& c, int32_t entry) {
  return static_cast<uint32_t>(entry) < static_cast<uint32_t>(c.pages) ? entry : -1;
}

// Index of (page, head, position) among the pool's token slots: times 64 or 128 for its code
// bytes, times 4 for its parameters.
SQ_HOST_DEVICE int64_t token_slot(const PagedCache& c, int32_t page, int32_t head, int64_t pos) {
  return ((static_cast<int64_t>(page) * c.heads + head) << c.shift) + (pos & ((int64_t{1} << c.shift) - 1));
}

// The tokens that rows of a sequence see, as one run of `tokens` places: the first `head` tokens, then those
// from `start` on.  Both are whole blocks of 64, so that a block of the run is one of the sequence.
struct TokenRun {
  int32_t head, start, tokens;
  SQ_HOST_DEVICE int32_t position(int32_t place) const { return place < head ? place : place - head + start; }
};

// That of rows whose earliest position is `low` and which see no token from `end` on (base + i + 1 of the
// last row of a chain, the length where a mask decides).  window 0: all tokens.
SQ_HOST_DEVICE TokenRun token_run(int32_t low, int32_t end, int32_t window, int32_t sinks) {
  constexpr int32_t kWhole = ~63;
  if (end < 0) end = 0;
  const int32_t from = low - window + 1, head = (sinks + 63) & kWhole;
  const int32_t start = window > 0 && from > 0 ? from & kWhole : 0;
  if (start <= head) return {0, 0, end};
  if (end <= start) return {0, 0, end < head ? end : head};
  return {head, start, head + (end - start)};
}

}  // namespace sq
