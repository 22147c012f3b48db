// The small kernels around a step on the paged cache: pages back to the pool and out of it, masks of a tree of
// drafts, and the move of the accepted ones.  All but the last touch a few kilobytes: what they cost is a
// launch and a chain of trips to memory, so each keeps that chain short.
//
// paged_release and paged_grow run in one workgroup, since the place of a page in the pool is a sum over all
// sequences before it.  Sequences come in batches of one for each thread; a batch's sums (a scan) stay in
// LDS, and its pages, or rows, are then taken evenly by the threads, each finding its sequence by halving.
//
// Measured on the device, us (an empty kernel takes 2): release 3.8 for 8 sequences, 7.7 for 256 of which 64 end;
// grow 4.8 and 6.2; the 36 000 rows of the latter step 4.4; masks of 8 and 16 trees 2.5 and 5.1;
// the accepted drafts of one sequence 3.2, of 64 sequences of 8 heads 3.3.  Eager calls wait for the host: 8 us for
// one, 17 for the two of a step's tables.
// A release looks at every block of its ranges, 1024 in 1.6 us.  64 sequences behind windows of 4096 tokens, pages of 16:
// 3.9 us with `first` from the last end, whatever the length; from the first tokens 28 at 8192 tokens and 800 at 131072.
#include "paged_device.h"
#include "sq_internal.h"

namespace sq {
namespace {

constexpr int kPoolThreads = 1024;
constexpr int kPoolWaves = kPoolThreads / 64;
constexpr int64_t kMost32 = 2147483647;

// Exclusive sums of v over the threads of the workgroup, and the sum of all; `slots` is scratch of one use.
struct Scan {
  int64_t before, all;
};
__device__ __forceinline__ Scan group_scan(int64_t v, int64_t* slots) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t upto = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) slots[w] = upto;
  __syncthreads();
  int64_t before = upto - v, all = 0;
#pragma unroll
  for (int x = 0; x < kPoolWaves; ++x) {
    const int64_t o = slots[x];
    if (x < w) before += o;
    all += o;
  }
  return {before, all};
}

// The last of n ascending values that is <= x (before[0] <= x).
template <typename V>
__device__ __forceinline__ int last_upto(const V* before, int n, V x) {
  int lo = 0, hi = n;  // before[lo] <= x < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int64_t blocks_of(int64_t tokens, int shift) { return (tokens + (int64_t{1} << shift) - 1) >> shift; }

__global__ void __launch_bounds__(kPoolThreads)
paged_release(const int32_t* first, const int32_t* end, PoolArgs p) {
  __shared__ int64_t before[kPoolThreads];  // blocks of the batch's sequences before each
  __shared__ int32_t from[kPoolThreads];    // first block of each that goes
  __shared__ int64_t slots[2][kPoolWaves];
  const int64_t free = min(max(p.count[0], 0), p.pages);
  int64_t back = 0;  // pages that went so far
  int turn = 0;
  for (int64_t b0 = 0; b0 < p.B; b0 += kPoolThreads) {
    const int64_t b = b0 + threadIdx.x;
    const int n = static_cast<int>(min(p.B - b0, static_cast<int64_t>(kPoolThreads)));
    int64_t blocks = 0;
    if (b < p.B) {
      const int32_t f = max(first[b], 0), e = end[b], held = p.held[b], have = min(max(held, 0), p.cols);
      const int64_t c0 = min(blocks_of(f, p.shift), static_cast<int64_t>(have));
      const bool to_end = e >= static_cast<int64_t>(have) << p.shift;
      const int64_t c1 = to_end ? have : max(e, 0) >> p.shift;
      blocks = max(c1 - c0, int64_t{0});
      from[threadIdx.x] = static_cast<int32_t>(c0);
      const int32_t now = to_end ? static_cast<int32_t>(c0) : have;
      if (now != held) p.held[b] = now;
    }
    const Scan s = group_scan(blocks, slots[turn ^= 1]);
    before[threadIdx.x] = s.before;
    __syncthreads();
    for (int64_t x0 = 0; x0 < s.all; x0 += kPoolThreads) {
      const int64_t x = x0 + threadIdx.x;
      int32_t page = -1;
      if (x < s.all) {
        const int k = last_upto(before, n, x);
        int32_t* const entry = p.table + (b0 + k) * p.ldt + from[k] + (x - before[k]);
        page = *entry;
        *entry = -1;
      }
      const bool good = static_cast<uint32_t>(page) < static_cast<uint32_t>(p.pages);
      const Scan at = group_scan(good, slots[turn ^= 1]);
      const int64_t place = free + back + at.before;
      if (good && place < p.pages) p.pool[place] = page;
      back += at.all;
    }
    __syncthreads();
  }
  // (each thread has read count before the scans' barriers)
  if (threadIdx.x == 0) p.count[0] = static_cast<int32_t>(min(free + back, static_cast<int64_t>(p.pages)));
}

// Slot of position pos of sequence b, -1 where the table has none.
__device__ __forceinline__ int64_t slot_of(const PoolArgs& p, int64_t b, int64_t pos) {
  const int64_t col = pos >> p.shift;
  if (pos < 0 || col >= p.cols) return -1;
  const int32_t page = p.table[b * p.ldt + col];
  if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.pages)) return -1;
  return (static_cast<int64_t>(page) << p.shift) + (pos & ((int64_t{1} << p.shift) - 1));
}

// Up to this many rows are written down by the workgroup that hands out the pages; more by a kernel behind it.
constexpr int64_t kRowsHere = 2 * kPoolThreads;

__global__ void __launch_bounds__(kPoolThreads)
paged_grow(PoolArgs p, GrowArgs g) {
  __shared__ int64_t pages_before[kPoolThreads], rows_before[kPoolThreads];
  __shared__ int32_t from[kPoolThreads], had[kPoolThreads];
  __shared__ int64_t slots[2][kPoolWaves];
  __shared__ unsigned long long columns;  // that the table lacks
  const int64_t free = min(max(p.count[0], 0), p.pages);
  int turn = 0;
  // what sequence b asks for
  struct Need {
    int32_t have, add, held, pages;
    int64_t columns;  // beyond the table
  };
  const auto need_of = [&](int64_t b) -> Need {
    if (b >= p.B) return {0, 0, 0, 0, 0};
    const int32_t have = max(g.have[b], 0), held = min(max(p.held[b], 0), p.cols);
    const int64_t tokens = min(static_cast<int64_t>(have) + max(g.add[b], 0), kMost32);
    const int64_t upto = blocks_of(tokens, p.shift);
    return {have, static_cast<int32_t>(tokens - have), held, static_cast<int32_t>(max(min(upto, static_cast<int64_t>(p.cols)) - held, int64_t{0})),
            max(upto - p.cols, int64_t{0})};
  };
  // All or nothing: the sums over all sequences first.  (With one batch they are the sums that it goes by.)
  Need mine = need_of(threadIdx.x);
  Scan pages{0, 0}, rows{0, 0};
  int64_t all_pages = 0, all_rows = 0;
  if (threadIdx.x == 0) columns = 0;
  for (int64_t b0 = 0; b0 < p.B || b0 == 0; b0 += kPoolThreads) {
    const Need n = b0 == 0 ? mine : need_of(b0 + threadIdx.x);
    const Scan sp = group_scan(n.pages, slots[turn ^= 1]);
    if (n.columns) atomicAdd(&columns, static_cast<unsigned long long>(n.columns));  // (whole numbers: in any order)
    const Scan sr = group_scan(n.add, slots[turn ^= 1]);
    if (b0 == 0) {
      pages = sp;
      rows = sr;
    }
    all_pages += sp.all;
    all_rows += sr.all;
  }
  const int64_t lack = max(all_pages - free, int64_t{0}) + static_cast<int64_t>(columns), over = max(all_rows - g.T, int64_t{0});
  const bool fine = lack == 0 && over == 0;
  if (threadIdx.x == 0) {
    g.missing[0] = static_cast<int32_t>(min(lack, kMost32));
    g.missing[1] = static_cast<int32_t>(min(over, kMost32));
    g.cu[0] = 0;
    if (fine) p.count[0] = static_cast<int32_t>(free - all_pages);
  }
  const bool here = g.T <= kRowsHere;
  if (!fine) {
    for (int64_t b = threadIdx.x; b < p.B; b += kPoolThreads) {
      g.lens[b] = max(g.have[b], 0);
      g.cu[b + 1] = 0;
    }
    if (here)
      for (int64_t t = threadIdx.x; t < g.T; t += kPoolThreads) {
        g.pos[t] = -1;
        g.slots[t] = -1;
      }
    return;
  }
  int64_t out = 0, row0 = 0;  // pages and rows of the batches before
  for (int64_t b0 = 0; b0 < p.B; b0 += kPoolThreads) {
    const int64_t b = b0 + threadIdx.x;
    const int n = static_cast<int>(min(p.B - b0, static_cast<int64_t>(kPoolThreads)));
    if (b0 > 0) {
      mine = need_of(b);
      pages = group_scan(mine.pages, slots[turn ^= 1]);
      rows = group_scan(mine.add, slots[turn ^= 1]);
    }
    if (b < p.B) {
      g.lens[b] = mine.have + mine.add;
      g.cu[b + 1] = static_cast<int32_t>(row0 + rows.before + mine.add);
      p.held[b] = mine.held + mine.pages;
    }
    pages_before[threadIdx.x] = pages.before;
    rows_before[threadIdx.x] = rows.before;
    from[threadIdx.x] = mine.held;
    had[threadIdx.x] = mine.have;
    __syncthreads();
    for (int64_t x = threadIdx.x; x < pages.all; x += kPoolThreads) {
      const int k = last_upto(pages_before, n, x);
      p.table[(b0 + k) * p.ldt + from[k] + (x - pages_before[k])] = p.pool[free - 1 - out - x];
    }
    __syncthreads();  // (the rows' slots read what the threads have written)
    if (here)
      for (int64_t x = threadIdx.x; x < rows.all; x += kPoolThreads) {
        const int k = last_upto(rows_before, n, x);
        const int64_t pos = had[k] + (x - rows_before[k]), t = row0 + x;
        g.pos[t] = static_cast<int32_t>(pos);
        g.slots[t] = slot_of(p, b0 + k, pos);
      }
    out += pages.all;
    row0 += rows.all;
    __syncthreads();
  }
  if (here)
    for (int64_t t = row0 + threadIdx.x; t < g.T; t += kPoolThreads) {
      g.pos[t] = -1;
      g.slots[t] = -1;
    }
}

// The rows of a large step behind paged_grow: 256 of them a workgroup.
__global__ void __launch_bounds__(256)
paged_rows(PoolArgs p, GrowArgs g) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (t >= g.T) return;
  int64_t pos = -1, slot = -1;
  if (t < g.cu[p.B]) {
    // the sequence with cu[b] <= t < cu[b + 1]: the last with cu[b] <= t has rows
    int64_t lo = 0, hi = p.B;
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) >> 1;
      if (g.cu[mid] <= t)
        lo = mid;
      else
        hi = mid;
    }
    pos = static_cast<int64_t>(g.lens[lo]) - g.cu[lo + 1] + t;
    slot = slot_of(p, lo, pos);
  }
  g.pos[t] = static_cast<int32_t>(pos);
  g.slots[t] = slot;
}

// A workgroup per sequence, a thread per draft: up the tree by the parents, which lie in LDS.  The way up is as long as
// the draft is deep, so a sequence has kMaskDrafts of them at most; those behind are written down as unseeing.
constexpr int kMaskThreads = 128;

__global__ void __launch_bounds__(kMaskThreads)
tree_mask(const int32_t* parents, const int32_t* cu, const int32_t* lens, int64_t b_first, TreeMaskArgs a) {
  __shared__ int16_t up[kMaskDrafts];  // -1: a root
  const int64_t b = b_first + blockIdx.x;
  const int most = static_cast<int>(a.T);
  const int q0 = min(max(cu[b], 0), most), all = max(min(cu[b + 1], most) - q0, 0), n = min(all, kMaskDrafts);
  const int base = lens ? min(max(lens[b], 0), (1 << 30) - 1) - all : 0;
  for (int i = threadIdx.x; i < n; i += kMaskThreads) {
    const int p = parents[q0 + i];
    up[i] = static_cast<int16_t>(p >= 0 && p < i ? p : -1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kMaskThreads) {
    int depth = 0;
    for (int j = up[i]; j >= 0; j = up[j]) ++depth;
    a.depth[q0 + i] = depth;
    int32_t* const row = a.mask + static_cast<int64_t>(q0 + i) * a.ldm;
    int j = i, d = depth;
    // two words at a time, from the last that has a bit down: parents come before their children
    for (int pair = (a.words - 1) / 2; pair >= 0; --pair) {
      uint64_t bits = 0;
      for (; j >= 64 * pair; j = up[j], --d)
        if (j < 64 * (pair + 1) && (a.window == 0 || depth - d < a.window || base + d < a.sinks)) bits |= uint64_t{1} << (j - 64 * pair);
      row[2 * pair] = static_cast<int32_t>(bits);
      if (2 * pair + 1 < a.words) row[2 * pair + 1] = static_cast<int32_t>(bits >> 32);
    }
  }
  for (int64_t i = n + static_cast<int64_t>(threadIdx.x); i < all; i += kMaskThreads) {
    a.depth[q0 + i] = 0;
    for (int x = 0; x < a.words; ++x) a.mask[(q0 + i) * a.ldm + x] = 0;
  }
}

// One workgroup per (sequence, head): 16 lanes an entry of the path, 16 entries at a time.  All of them are read
// before any is written, and an entry's draft lies at or behind its place, so that no draft is lost.
constexpr int kKeepThreads = 256;
constexpr int kKeepEntries = kKeepThreads / 16;

template <int BITS, bool P16>
__global__ void __launch_bounds__(kKeepThreads)
kv_keep(const int32_t* cu, const int32_t* lens, const int32_t* path, const int32_t* kept, int64_t group_first, uint32_t magic_heads,
        KeepArgs a) {
  constexpr int ROW = BITS * 16, UNITS = ROW / 16;  // 16-byte pieces of a token's codes
  const int lane = threadIdx.x & 15;
  // (heads below 2^16 and a part of the grid below 2^24 groups: 32 bits)
  uint32_t seq, head;
  div_rem(blockIdx.x, a.cache.heads, magic_heads, seq, head);
  const int64_t b = group_first + seq;
  const int64_t n = max(static_cast<int64_t>(cu[b + 1]) - cu[b], int64_t{0});
  const int64_t base = static_cast<int64_t>(lens[b]) - n;
  const int64_t count = min(static_cast<int64_t>(min(max(kept[b], 0), a.most)), n);
  if (head == 0 && threadIdx.x == 0) a.lens_out[b] = static_cast<int32_t>(max(base + count, int64_t{0}));
  const int32_t* const table = a.cache.table + b * a.cache.ldt;
  const auto slot = [&](int64_t pos) -> int64_t {
    const int32_t col = table_column(a.cache, pos);
    if (col < 0) return -1;
    const int32_t page = valid_page(a.cache, table[col]);
    return page < 0 ? -1 : token_slot(a.cache, page, head, pos);
  };
  for (int64_t e0 = 0; e0 < count; e0 += kKeepEntries) {
    const int64_t e = e0 + (threadIdx.x >> 4);
    int64_t from = -1, to = -1;
    if (e < count) {
      const int32_t draft = path[b * a.ldp + e];
      if (draft > e && draft < n) {  // (a draft that is in its place already stays)
        from = slot(base + draft);
        to = slot(base + e);
      }
    }
    const bool moves = from >= 0 && to >= 0;
    // 4 bits: lanes 0 .. 3 keys, 4 .. 7 values, 8 parameters; 8 bits: 0 .. 7, 8 .. 15, and parameters with lane 0
    uint8_t* const codes = lane < UNITS ? a.cache.kq : a.cache.vq;
    const int piece = 16 * (lane & (UNITS - 1));
    const bool code_lane = lane < 2 * UNITS, param_lane = lane == (UNITS == 4 ? 8 : 0);
    v4u c = {0, 0, 0, 0}, p = {0, 0, 0, 0};
    if (moves) {
      if (code_lane) c = *reinterpret_cast<const v4u*>(codes + from * ROW + piece);
      if (param_lane) {
        if constexpr (P16) {
          const v2u h = static_cast<const v2u*>(a.cache.params)[from];
          p[0] = h[0];
          p[1] = h[1];
        } else {
          p = static_cast<const v4u*>(a.cache.params)[from];
        }
      }
    }
    __syncthreads();
    if (moves) {
      if (code_lane) *reinterpret_cast<v4u*>(codes + to * ROW + piece) = c;
      if (param_lane) {
        if constexpr (P16)
          static_cast<v2u*>(a.cache.params)[to] = v2u{p[0], p[1]};
        else
          static_cast<v4u*>(a.cache.params)[to] = p;
      }
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_paged_release(const PoolArgs& p, const int32_t* first, const int32_t* end, hipStream_t stream) {
  return launch(paged_release, dim3(1), dim3(kPoolThreads), 0, stream, first, end, p);
}

hipError_t launch_paged_grow(const PoolArgs& p, const GrowArgs& g, hipStream_t stream) {
  const hipError_t e = launch(paged_grow, dim3(1), dim3(kPoolThreads), 0, stream, p, g);
  if (e != hipSuccess || g.T <= kRowsHere) return e;
  return launch(paged_rows, dim3(static_cast<unsigned>((g.T + 255) / 256)), dim3(256), 0, stream, p, g);
}

hipError_t launch_tree_mask(const TreeMaskArgs& a, hipStream_t stream) {
  return in_parts(a.B, max_blocks(kMaskThreads), [&](int64_t b, int64_t n) {
    return launch(tree_mask, dim3(static_cast<unsigned>(n)), dim3(kMaskThreads), 0, stream, a.parents, a.cu, a.lens, b, a);
  });
}

hipError_t launch_kv_keep(const KeepArgs& a, hipStream_t stream) {
  return in_parts(a.B, max_blocks(kKeepThreads) / a.cache.heads, [&](int64_t b, int64_t n) {
    const auto go = [&](auto kern) {
      return launch(kern, dim3(static_cast<unsigned>(n * a.cache.heads)), dim3(kKeepThreads), 0, stream, a.cu, a.lens, a.path, a.kept, b,
                    div_magic(static_cast<uint32_t>(a.cache.heads)), a);
    };
    if (a.bits == 8) return a.param16 ? go(kv_keep<8, true>) : go(kv_keep<8, false>);
    return a.param16 ? go(kv_keep<4, true>) : go(kv_keep<4, false>);
  });
}

}  // namespace sq
