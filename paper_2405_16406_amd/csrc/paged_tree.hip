// Attention of a sequence's last tokens over its pages (paged_attn.hip has the mathematics of one row): drafts
// of a tree, each with the drafts that it sees as bits, or a chain of tokens; and of single tokens with a
// window.  Row (i, h) of a sequence, i < n its token and h a query head of the key/value head, sees
//     mask:   t < base where t > base + depth_i - window or t < sinks, and the drafts base + j of its bits
//     chain:  t <= base + i with the same window at base + i.
//
// A workgroup of four or eight waves serves one (sequence, key/value head, 16 RB of its rows, chunk of the tokens that
// these rows see); its waves take the chunk's blocks of 64 tokens in turn, each on its own.  A block's codes
// become operands once for all RB columns of 16 rows.  What a row does not see is cut out of the scores by
// 16 bits a lane, one for each of its tokens, in the blocks alone that some row does not see whole.
//
// Many rows: vector instructions bound it.  64 drafts of 32 heads on 8 behind 131008 tokens of 4 bits take 200 us with
// the join (137 GFLOP, 0.69 PFLOP/s of the 1.49 that a large library product reaches; the cache's 150 MB alone would
// take 30): 566 vector operations for 64 tokens and two columns, a third of them the codes' expansion (80 of the keys, 112
// of the values), half the softmax, keep the vector units in use for 78 % of the kernel's cycles, the matrix cores for 30 %.  More rows on an
// expansion: four columns a wave need 512 registers and spilled (413 us, two columns then 227); workgroups of 128 rows
// that share the operands through LDS took 213 then, and 107 with 16 sequences of 524 .. 8224 tokens, 64 heads on 8,
// where two columns a wave took 70 (62 now).
// Few rows: memory.  64 sequences' windows of 2048 tokens, 115 MB, 31 us (3.7 TB/s; three waves a SIMD, which spill four
// registers, 41, and 50 with workgroups of six); 4 drafts behind those 131008
// tokens 38 with the join.  Short runs: two launches and their chains to memory (16 drafts behind 2048 tokens 10 us,
// the join 4).
#include "paged_attn_device.h"

namespace sq {
namespace {

// Sequence and tile of rows of the tile number `rem` among ceil(n * group / ROWS) a sequence; seq -1: past the last.
struct TreeTile {
  int seq, tile;
  int q0, n, len;
};
template <int ROWS>
__device__ __forceinline__ TreeTile find_tree_tile(const int32_t* cu, const int32_t* lens, int64_t B, int64_t T, int group, int rem) {
  if (!cu) {
    const int per = (group + ROWS - 1) / ROWS;
    const int b = rem / per;
    return {b, rem - b * per, b, 1, lens[b]};
  }
  const int lane = threadIdx.x & 63;
  for (int64_t b0 = 0; b0 < B; b0 += 64) {
    int q0 = 0, n = 0, len = 0;
    if (b0 + lane < B) {  // clamped to the rows, whatever cu holds
      const int most = static_cast<int>(T);
      const int first = cu[b0 + lane], end = cu[b0 + lane + 1];
      len = lens[b0 + lane];
      q0 = min(max(first, 0), most);
      n = max(min(end, most) - q0, 0);
    }
    const int tiles = (n * group + ROWS - 1) / ROWS;
    const int upto = wave_scan(tiles);
    const uint64_t past = __ballot(upto > rem);
    if (past) {
      const int f = __builtin_ctzll(past);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
      return {static_cast<int>(b0) + f, rem - (of(upto) - of(tiles)), of(q0), of(n), of(len)};
    }
    rem -= __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, 0, 0, 0};
}

// Bits x of a block's tokens t .. t + 63 with t + x < end.
__device__ __forceinline__ uint64_t below(int end, int t) {
  const int n = min(max(end - t, 0), kBlock);
  return n == kBlock ? ~uint64_t{0} : (uint64_t{1} << n) - 1;
}
// Of a block's 64 bits those of a lane's 16 tokens 16 j + 4 g + r, in the order of its scores, 4 j + r.
__device__ __forceinline__ uint32_t lane_bits(uint64_t block) {
  const uint64_t mine = block >> (4 * ((threadIdx.x & 63) >> 4));
  const auto four = [&](int j) { return static_cast<uint32_t>(mine >> (16 * j)) & 0xFu; };
  return four(0) | four(1) << 4 | four(2) << 8 | four(3) << 12;
}

// What a workgroup has to do: its tile of rows, and of the run of tokens that these see the places first .. last - 1.
struct TreePlace {
  int seq, q0, n;    // the sequence, its first row of the call and its rows
  int base, len;     // tokens before the rows; tokens that count
  int r0, rows;      // first row of the tile (16 RB .. of them), rows of the sequence
  TokenRun run;
  int first, last;
  int c, own;        // the chunk, and how many the tile has
  int hk;
  const int32_t* table;
};

// false: nothing (the workgroup leaves together).  Workgroups in the order of dispatch as in attn_paged_part: the
// chunks from a tile's last one back slowest, then tile, then key/value head (so that the tiles which share keys
// follow each other on one of the chip's caches).
template <int ROWS>
__device__ __forceinline__ bool find_place(const int32_t* cu, const int32_t* lens, uint32_t magic_tiles, uint32_t magic_heads,
                                           uint32_t magic_group, const TreeArgs& a, TreePlace& p) {
  uint32_t rest, hk, back, number;
  div_rem(blockIdx.x, a.cache.heads, magic_heads, rest, hk);
  div_rem(rest, a.plan.tiles, magic_tiles, back, number);
  back = a.plan.chunks - 1 - back;
  const TreeTile tt = find_tree_tile<ROWS>(cu, lens, a.B, a.T, a.group, static_cast<int>(number));
  if (tt.seq < 0) return false;
  const int all = min(max(tt.len, 0), (1 << 30) - 1);  // (a position plus a depth stays below 2^31)
  p.seq = tt.seq;
  p.q0 = tt.q0;
  p.n = tt.n;
  p.base = all - tt.n;
  p.len = min(all, a.max_len);
  p.rows = tt.n * a.group;
  p.r0 = tt.tile * ROWS;
  p.hk = static_cast<int>(hk);
  const auto token_of = [&](int r) {
    uint32_t t, h;
    div_rem(static_cast<uint32_t>(r), a.group, magic_group, t, h);
    return static_cast<int>(t);
  };
  const int i0 = token_of(p.r0), i1 = token_of(min(p.r0 + ROWS, p.rows) - 1);  // first and last token of the tile
  p.run = token_run(a.mask ? p.base : p.base + i0, a.mask ? p.len : min(p.base + i1 + 1, p.len), a.window, a.sinks);
  p.own = max(1, (p.run.tokens + a.plan.chunk_tokens - 1) / a.plan.chunk_tokens);
  if (static_cast<int>(back) >= p.own) return false;
  p.c = p.own - 1 - static_cast<int>(back);
  p.first = p.c * a.plan.chunk_tokens;
  p.last = min(p.run.tokens, p.first + a.plan.chunk_tokens);
  p.table = a.cache.table + tt.seq * a.cache.ldt;
  return true;
}

// The table's entry of the 16 tokens of a block (at place v0 of the run) that lane / 16 stands for.
__device__ __forceinline__ int32_t entry_of(const TreeArgs& a, const TreePlace& p, int v0) {
  if (v0 >= p.last) return -1;
  const int32_t col = table_column(a.cache, p.run.position(v0) + 16 * ((threadIdx.x & 63) >> 4));
  return col < 0 ? -1 : p.table[col];
}

// Parameters of the token in slot `slot` of the pool.
template <bool P16>
__device__ __forceinline__ float4 token_params(const PagedCache& c, int64_t slot) {
  if constexpr (P16) {
    const uint2 p = static_cast<const uint2*>(c.params)[slot];
    return make_float4(h2f(static_cast<uint16_t>(p.x)), h2f(static_cast<uint16_t>(p.x >> 16)), h2f(static_cast<uint16_t>(p.y)),
                       h2f(static_cast<uint16_t>(p.y >> 16)));
  } else {
    return static_cast<const float4*>(c.params)[slot];
  }
}

// Coefficients of a block's 64 tokens, one a lane, in rows of 64: a, b, lv, 1 / va and vb / va with the score
// s_t + log2 va_t = a_t (q . c_t) + b_t sum(q) + lv_t, as in paged_attn.hip.  A weight of 0 does not hide a
// 1 / va or vb / va that is not finite: such tokens (the result) have zeros there, and what they are in
// rows 5 and 6.  With rows that are scaled apart lv is in row 7, and the third has 0 in its place.
__device__ __forceinline__ uint64_t token_coefs(float4 par, bool there, float cs, float down, bool apart, float* coef) {
  const int lane = threadIdx.x & 63;
  par.z = par.z == 0.0f ? 1.0f : par.z;  // a slot of a zeroed cache that was never written
  float rva = there ? __fdiv_rn(1.0f, par.z) : 0.0f, rvb = there ? par.w * rva : 0.0f;
  const bool bad = !(fabsf(rva) < INFINITY) || !(fabsf(rvb) < INFINITY);
  const uint64_t odd = __ballot(bad);
  float lv = there ? __builtin_amdgcn_logf(par.z) : -INFINITY;
  if (__builtin_expect(odd != 0 || apart, 0)) {
    coef[5 * kBlock + lane] = rva;
    coef[6 * kBlock + lane] = rvb;
    if (bad) rva = rvb = 0.0f;
    if (apart) {
      coef[7 * kBlock + lane] = lv;
      lv = there ? 0.0f : -INFINITY;
    }
  }
  coef[0 * kBlock + lane] = there ? par.x * (cs * 16777216.0f * down) : 0.0f;  // 2^24 undoes the codes' subnormal scale
  coef[1 * kBlock + lane] = there ? par.y * cs : 0.0f;
  coef[2 * kBlock + lane] = lv;
  coef[3 * kBlock + lane] = rva;
  coef[4 * kBlock + lane] = rvb;
  return odd;
}

// A token's key codes of dims 32 g .. 32 g + 31 as the four operands of a lane (4 bits: odd dims in place, 16 n, for
// queries that have 1 / 16 there).
template <int BITS, int KW>
__device__ __forceinline__ void key_operands(const v4u (&k)[KW], v8h (&ko)[4]) {
  if constexpr (BITS == 4) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t u = k[0][2 * e], v = k[0][2 * e + 1];
      ko[2 * e] = operand(u & 0x000F000Fu, (u >> 8) & 0x000F000Fu, v & 0x000F000Fu, (v >> 8) & 0x000F000Fu);
      ko[2 * e + 1] = operand(u & 0x00F000F0u, (u >> 8) & 0x00F000F0u, v & 0x00F000F0u, (v >> 8) & 0x00F000F0u);
    }
  } else {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const uint32_t u = k[x / 2][2 * (x & 1)], v = k[x / 2][2 * (x & 1) + 1];
      ko[x] = operand(u & 0x00FF00FFu, (u >> 8) & 0x00FF00FFu, v & 0x00FF00FFu, (v >> 8) & 0x00FF00FFu);
    }
  }
}

// Two of four codes of 4 bits, a byte each, as the numbers normal() makes: n is the 8-bit float (e4m3) of n 2^-9, and its
// conversion exact, a mask and a product less for a pair (64 drafts behind 131008 tokens: 225 -> 219 us).
template <bool HIGH>
__device__ __forceinline__ uint32_t normal_pair(uint32_t bytes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(bytes), 1.0f, HIGH));
}

// Value codes of a block in LDS, a token's 16 bytes apart from the next one's (so that a read's place is one register
// and a constant; paged_attn.hip's exchanged units would take a register for each): dims 16 dt + i of the lane's 16
// tokens as two operands.
template <int BITS>
constexpr int kPitch = BITS * 16 + 16;
template <int BITS>
__device__ __forceinline__ void value_operands(const uint8_t* codes, int dt, v8h (&vo)[2]) {
  typedef __attribute__((address_space(3))) v2i* lds_v2i;
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  if constexpr (BITS == 4) {
    const int row = 16 * (i >> 2) + 4 * g + (i & 3);  // the lane's i-th token
    const v2i c2 = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_v2i)(uintptr_t)(codes + row * kPitch<BITS> + 8 * dt));
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t even = static_cast<uint32_t>(c2[x]) & 0x0F0F0F0Fu, odd = (static_cast<uint32_t>(c2[x]) >> 4) & 0x0F0F0F0Fu;
      vo[x] = operand(normal_pair<false>(even), normal_pair<true>(even), normal_pair<false>(odd), normal_pair<true>(odd));
    }
  } else {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int n = 8 * x + (i >> 1), row = 16 * (n >> 2) + 4 * g + (n & 3);  // its n-th
      const v2i c2 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(uintptr_t)(codes + row * kPitch<BITS> + 16 * dt + 8 * (i & 1)));
      const uint32_t u = static_cast<uint32_t>(c2[0]), v = static_cast<uint32_t>(c2[1]);
      vo[x] = operand(normal(u & 0x00FF00FFu, 0), normal((u >> 8) & 0x00FF00FFu, 0), normal(v & 0x00FF00FFu, 0),
                      normal((v >> 8) & 0x00FF00FFu, 0));
    }
  }
}

// 16 RB rows of a wave, one a lane and column: queries, what they see, and their softmax states.
template <int BITS, int RB>
struct TreeRows {
  v8h qf[RB][4];    // dims 32 g .. 32 g + 31 in the codes' pair order, divided by `down` (4 bits: odd dims 1 / 16 of that)
  float down;
  bool apart;       // each row is divided by its own number instead, and down is 1
  float qsum[RB];   // sums over all dims, divided alike with `apart`
  int lo_most, hi_least;  // every row sees t where lo_most <= t < hi_least (or t < sinks)
  int* sight;       // in LDS, out of the registers: [hi, lo, row, and with `apart` its divisor][16] of each column
  float m[RB], l[RB], bsum[RB];
  uint32_t seen;    // bit rb: the row sees a token with a page
  v4f acc[RB][8];

  static constexpr int KIND = BITS == 4 ? 4 : 3, SIGHT = KIND * 16 * RB;  // numbers in LDS

  // The exponent of the power of two that brings a number of this size to 2^13 .. 2^14; 0 for 0 and what is not finite.
  static __device__ __forceinline__ int lift(float size) {
    return size > 0.0f && size < INFINITY ? 13 + 127 - static_cast<int>(__float_as_uint(size) >> 23) : 0;
  }
  static __device__ __forceinline__ float power(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }

  // Rows p.r0 + 16 rb + i; past the last: that one again, not stored.
  __device__ __forceinline__ void init(const uint16_t* q, uint32_t magic_group, const TreeArgs& a, const TreePlace& p, int* in_lds) {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    sight = in_lds;
    seen = 0;
    lo_most = 0;
    hi_least = p.len;
    float size[RB];  // of the largest of the lane's 32 elements of the row (NaN left out)
    v4u all[RB][4];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m[rb] = -INFINITY;
      l[rb] = bsum[rb] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[rb][dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      uint32_t tok, gh;
      div_rem(static_cast<uint32_t>(min(p.r0 + 16 * rb + i, p.rows - 1)), a.group, magic_group, tok, gh);
      const int64_t t = p.q0 + static_cast<int64_t>(tok);
      const v4u* qv = reinterpret_cast<const v4u*>(q + t * a.ldq + (static_cast<int64_t>(p.hk) * a.group + gh) * 128 + 32 * g);
      v4u raw[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) raw[x] = qv[x];
      int at = static_cast<int>(tok);
      if (a.mask && a.depth && a.window > 0) at = min(max(a.depth[t], 0), 1 << 30);
      const int hi = min(a.mask ? p.base : p.base + static_cast<int>(tok) + 1, p.len);
      const int lo = a.window > 0 ? max(p.base + at - a.window + 1, 0) : 0;
      hi_least = min(hi_least, hi);
      lo_most = max(lo_most, lo);
      if (g == 0) {
        sight[(KIND * rb + 0) * 16 + i] = hi;
        sight[(KIND * rb + 1) * 16 + i] = lo;
        sight[(KIND * rb + 2) * 16 + i] = static_cast<int>(t);  // (rows below 2^24)
      }
      float sum = 0.0f;
      size[rb] = 0.0f;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float u = h2f(static_cast<uint16_t>(raw[x][y])), v = h2f(static_cast<uint16_t>(raw[x][y] >> 16));
          sum += u + v;
          size[rb] = fmaxf(size[rb], fmaxf(fabsf(u), fabsf(v)));
        }
      qsum[rb] = rows_all(sum, [](float u, float v) { return __fadd_rn(u, v); });
#pragma unroll
      for (int x = 0; x < 4; ++x) all[rb][x] = raw[x];
    }
    // 4 bits: the odd dims' sixteenth would lose bits of small numbers, so queries are first brought up to where the largest
    // lies in 2^13 .. 2^14, by a power of two.  What is rounded then (fp16's steps of 2^-24 at the low end) is 2^-34 of
    // the largest.  All rows of the wave share the power, which the coefficients undo, as long as that is 2^-24 or less
    // of what is largest in any lane's part of a row, a 32-bit rounding; else each has its own, undone in own_scales.
    // (Measured, us: 64 drafts of 32 heads behind 131008 tokens 192, with rows 2^-12 of the others among them 226; 16
    // sequences of 32 drafts of 64 heads behind 4096, 113 and 130.)
    down = 1.0f;
    apart = false;
    float up[RB];
    if constexpr (BITS == 4) {
      float most = 0.0f, least = INFINITY;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const bool counts = size[rb] > 0.0f && size[rb] < INFINITY;
        most = counts ? fmaxf(most, size[rb]) : most;
        least = counts ? fminf(least, size[rb]) : least;
      }
      most = wave_max(most);
      apart = __ballot(least < most * 0x1p-10f) != 0;
      if (__builtin_expect(apart, 0)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const int e = lift(rows_all(size[rb], [](float u, float v) { return fmaxf(u, v); }));
          up[rb] = power(e);
          qsum[rb] *= up[rb];
          if (g == 0) sight[(KIND * rb + 3) * 16 + i] = __float_as_int(power(-e));
        }
      } else {
        const int e = lift(most);
        down = power(-e);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) up[rb] = power(e);
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      v4u raw[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) raw[x] = all[rb][x];
      if constexpr (BITS == 4) {
        // (even dims in the low halves)
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y)
            raw[x][y] = f2h2(h2f(static_cast<uint16_t>(raw[x][y])) * up[rb], h2f(static_cast<uint16_t>(raw[x][y] >> 16)) * (0.0625f * up[rb]));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const v4u u = raw[2 * e], v = raw[2 * e + 1];
          qf[rb][2 * e] = operand(__builtin_amdgcn_perm(u[2], u[0], 0x05040100u), __builtin_amdgcn_perm(u[3], u[1], 0x05040100u),
                                  __builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x05040100u));
          qf[rb][2 * e + 1] = operand(__builtin_amdgcn_perm(u[2], u[0], 0x07060302u), __builtin_amdgcn_perm(u[3], u[1], 0x07060302u),
                                      __builtin_amdgcn_perm(v[2], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u));
        }
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          qf[rb][x] = operand(__builtin_amdgcn_perm(raw[x][1], raw[x][0], 0x05040100u), __builtin_amdgcn_perm(raw[x][1], raw[x][0], 0x07060302u),
                              __builtin_amdgcn_perm(raw[x][3], raw[x][2], 0x05040100u), __builtin_amdgcn_perm(raw[x][3], raw[x][2], 0x07060302u));
      }
    }
    // of all rows (lo and hi are not negative there but for hi of a base below 0, which counts as 0)
    lo_most = static_cast<int>(wave_all(static_cast<uint32_t>(lo_most), [](uint32_t u, uint32_t v) { return max(u, v); }));
    hi_least = static_cast<int>(wave_all(static_cast<uint32_t>(max(hi_least, 0)), [](uint32_t u, uint32_t v) { return min(u, v); }));
  }

  // Scores of the block's tokens 16 j + 4 g .. + 3 with their key operands.
  __device__ __forceinline__ void scores(int j, const v8h (&ko)[4], const float* coef, float (&s)[RB][16]) {
    const int g = (threadIdx.x & 63) >> 4;
    const float4 ca = *reinterpret_cast<const float4*>(coef + 0 * kBlock + 16 * j + 4 * g);
    const float4 cb = *reinterpret_cast<const float4*>(coef + 1 * kBlock + 16 * j + 4 * g);
    const float4 cl = *reinterpret_cast<const float4*>(coef + 2 * kBlock + 16 * j + 4 * g);
    const float fa[4] = {ca.x, ca.y, ca.z, ca.w}, fb[4] = {cb.x, cb.y, cb.z, cb.w}, fl[4] = {cl.x, cl.y, cl.z, cl.w};
    v4f dot[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) dot[rb] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) dot[rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ko[x], qf[rb][x], dot[rb], 0, 0, 0);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[rb][4 * j + r] = __fmaf_rn(fa[r], dot[rb][r], __fmaf_rn(fb[r], qsum[rb], fl[r]));
  }

  // With `apart`: scores of queries that each row has divided by its own number, without lv, to those of the queries.
  __device__ __forceinline__ void own_scales(const float* coef, float (&s)[RB][16]) const {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 cl = *reinterpret_cast<const float4*>(coef + 7 * kBlock + 16 * j + 4 * g);
      const float fl[4] = {cl.x, cl.y, cl.z, cl.w};
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float by = __int_as_float(sight[(KIND * rb + 3) * 16 + i]);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[rb][4 * j + r] = __fmaf_rn(s[rb][4 * j + r], by, fl[r]);
      }
    }
  }

  // Of the block's tokens t .. t + 63 those that the lane's row of column rb sees.
  __device__ __forceinline__ uint64_t visible(int rb, int t, const TreeArgs& a, const TreePlace& p) const {
    const int i = threadIdx.x & 15;
    const int hi = sight[(KIND * rb + 0) * 16 + i], lo = sight[(KIND * rb + 1) * 16 + i];
    uint64_t vis = below(hi, t) & (~below(lo, t) | below(a.sinks, t));
    if (a.mask && t + kBlock > p.base) {
      const int j = t - p.base, word = j >> 5, shift = j & 31;  // (rounded down: negative for the words before the first)
      const int32_t* const bits = a.mask + sight[(KIND * rb + 2) * 16 + i] * a.ldm;
      const auto at = [&](int x) { return x >= 0 && x < a.words ? static_cast<uint64_t>(static_cast<uint32_t>(bits[x])) : uint64_t{0}; };
      uint64_t sees = (at(word) | at(word + 1) << 32) >> shift;
      if (shift) sees |= at(word + 2) << (64 - shift);
      vis |= sees & below(min(p.base + p.n, p.len), t);
    }
    return vis;
  }

  // Takes what a row does not see out of the scores of the block at token t0.  there, odd: bits of its tokens that have
  // a page, and of those whose coefficients are not finite.
  __device__ __forceinline__ void hide(int t0, uint64_t there, uint64_t odd, const float* coef, const TreeArgs& a, const TreePlace& p,
                                       float (&s)[RB][16]) {
    const uint32_t here = lane_bits(there);  // of the lane's tokens
    const bool masked = t0 + kBlock > hi_least || (t0 < lo_most && t0 + kBlock > a.sinks);
    if (__builtin_expect(masked || odd != 0 || (BITS == 4 && apart), 0)) {
      if constexpr (BITS == 4)
        if (apart) own_scales(coef, s);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const uint32_t vis = masked ? lane_bits(visible(rb, t0, a, p)) : 0xFFFFu;
        seen |= static_cast<uint32_t>((vis & here) != 0) << rb;
#pragma unroll
        for (int x = 0; x < 16; ++x) {  // bitwise: a compare each would take the scalar registers' room
          const uint32_t keep = static_cast<uint32_t>(static_cast<int32_t>(vis << (31 - x)) >> 31);
          s[rb][x] = __uint_as_float((__float_as_uint(s[rb][x]) & keep) | (~keep & 0xFF800000u));  // -inf
        }
        // what the row sees of parameters that are not finite, whatever its weight
        for (uint32_t left = vis & lane_bits(odd); left; left &= left - 1) {
          const int k = __builtin_ctz(left), x = 16 * (k >> 2) + 4 * ((threadIdx.x & 63) >> 4) + (k & 3);
          const float r = coef[5 * kBlock + x], v = coef[6 * kBlock + x];
          if (!(fabsf(r) < INFINITY)) l[rb] += r;
          if (!(fabsf(v) < INFINITY)) bsum[rb] += v;
        }
      }
    } else if (here) {
      seen |= (1u << RB) - 1u;
    }
  }

  // Moves m, and what it scales, where the largest weight would grow too far (m = -inf: with any token).
  __device__ __forceinline__ void move(const float (&s)[RB][16]) {
    float top[RB];
    uint64_t moves = 0;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      top[rb] = s[rb][0];
#pragma unroll
      for (int x = 1; x < 16; ++x) top[rb] = fmaxf(top[rb], s[rb][x]);
      top[rb] = rows_all(top[rb], [](float u, float v) { return fmaxf(u, v); });
      moves |= __ballot(top[rb] - m[rb] > kWeightBits + kSlack);
    }
    if (__builtin_expect(moves != 0, 0)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const bool mine = top[rb] - m[rb] > kWeightBits + kSlack;
        const float mn = mine ? fmaxf(m[rb], fabsf(top[rb]) < kLargeScore ? top[rb] - kWeightBits : top[rb]) : m[rb];
        const float f = mine ? rescale(m[rb], mn) : 1.0f;
        // (what hide put there stays: f is 0 before the first token's weight)
        l[rb] = fabsf(l[rb]) < INFINITY ? l[rb] * f : l[rb];
        bsum[rb] = fabsf(bsum[rb]) < INFINITY ? bsum[rb] * f : bsum[rb];
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[rb][dt] *= f;
        m[rb] = mn;
      }
    }
  }

  // Weights of column rb in the value codes' pair order, rounded to fp16 as the second product takes them; l and b sum the
  // rounded ones, so that what a weight is off by moves the mean, not its size.  Outputs are then off by 2.3e-4 to
  // 2.8e-4 of their size, of which their own rounding is 2.1e-4.
  __device__ __forceinline__ void weights(int rb, const float (&s)[16], const float* coef, v8h (&pf)[2]) {
    const int g = (threadIdx.x & 63) >> 4;
    const float from = m[rb] == -INFINITY ? 0.0f : m[rb];
    uint32_t pw[8];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float4 cr0 = *reinterpret_cast<const float4*>(coef + 3 * kBlock + 32 * x + 4 * g);
      const float4 cr1 = *reinterpret_cast<const float4*>(coef + 3 * kBlock + 32 * x + 16 + 4 * g);
      const float4 cv0 = *reinterpret_cast<const float4*>(coef + 4 * kBlock + 32 * x + 4 * g);
      const float4 cv1 = *reinterpret_cast<const float4*>(coef + 4 * kBlock + 32 * x + 16 + 4 * g);
      const float fr[8] = {cr0.x, cr0.y, cr0.z, cr0.w, cr1.x, cr1.y, cr1.z, cr1.w};
      const float fv[8] = {cv0.x, cv0.y, cv0.z, cv0.w, cv1.x, cv1.y, cv1.z, cv1.w};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        // pairs of tokens: 4 bits (0, 2), (4, 6), (1, 3), (5, 7); 8 bits (0, 2), (1, 3), ..
        const int ta = BITS == 4 ? 4 * (y & 1) + (y >> 1) : 4 * (y >> 1) + (y & 1), tb = ta + 2;
        const uint32_t p2 = f2h2(exp2_fast(s[8 * x + ta] - from), exp2_fast(s[8 * x + tb] - from));
        pw[4 * x + y] = p2;
        const v2h ph = __builtin_bit_cast(v2h, p2);
        l[rb] = __fmaf_rn(static_cast<float>(ph[0]), fr[ta], l[rb]);
        l[rb] = __fmaf_rn(static_cast<float>(ph[1]), fr[tb], l[rb]);
        bsum[rb] = __fmaf_rn(static_cast<float>(ph[0]), fv[ta], bsum[rb]);
        bsum[rb] = __fmaf_rn(static_cast<float>(ph[1]), fv[tb], bsum[rb]);
      }
    }
    pf[0] = operand(pw[0], pw[1], pw[2], pw[3]);
    pf[1] = operand(pw[4], pw[5], pw[6], pw[7]);
  }

  __device__ __forceinline__ void values(int dt, const v8h (&vo)[2], const v8h (&pf)[RB][2]) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[rb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vo[x], pf[rb][x], acc[rb][dt], 0, 0, 0);
  }

  // The state of column rb when all blocks are through: l and b over all tokens, m as the join takes it.
  __device__ __forceinline__ void finish(int rb) {
    const auto add = [](float u, float v) { return __fadd_rn(u, v); };
    l[rb] = rows_all(l[rb], add);
    bsum[rb] = rows_all(bsum[rb], add);
    const float any = rows_all((seen >> rb) & 1u ? 1.0f : 0.0f, [](float u, float v) { return fmaxf(u, v); });
    if (any == 0.0f) {  // hidden tokens alone: a query that is not finite has made their sums NaN
      m[rb] = -INFINITY;
      l[rb] = bsum[rb] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[rb][dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    } else if (m[rb] == -INFINITY) {
      m[rb] = kNoScore;
    }
  }
};

// Puts down dims d .. d + 3 (not yet divided by L) of row `row` of the sequence: the output where the tile has one chunk,
// else the chunk's state.
__device__ __forceinline__ void store_row(const TreeArgs& a, const TreePlace& p, uint32_t magic_group, int row, int d, float M, float L, v4f D) {
  uint32_t tok, gh;
  div_rem(static_cast<uint32_t>(row), a.group, magic_group, tok, gh);
  if (a.cu && p.base + static_cast<int>(tok) < 0) return;  // a row without a place
  const int64_t t = p.q0 + static_cast<int64_t>(tok), head = static_cast<int64_t>(p.hk) * a.group + gh;
  float* pr = a.part + ((t * a.hq + head) * a.plan.chunks + p.c) * kAttnPart;
  if (a.plan.chunks > 1 && p.c == 0 && d == 0) pr[2] = static_cast<float>(p.own);  // what the join goes by
  if (p.own == 1) {
    uint16_t* o = a.out + t * a.ldo + head * 128 + d;
    if (M == -INFINITY)  // no token
      *reinterpret_cast<v2u*>(o) = v2u{0u, 0u};
    else
      *reinterpret_cast<v2u*>(o) = v2u{f2h2(__fdiv_rn(D[0], L), __fdiv_rn(D[1], L)), f2h2(__fdiv_rn(D[2], L), __fdiv_rn(D[3], L))};
  } else {
    if (d == 0) {
      pr[0] = M;
      pr[1] = L;
    }
    *reinterpret_cast<v4f*>(pr + 4 + d) = D;
  }
}

// LDS of a wave of attn_tree_part: value codes of a block, its coefficients, the rows' sight, their queries (with two
// columns, whose registers they would take).
template <int BITS, int RB>
struct TreeLds {
  static constexpr int CODES = kBlock * kPitch<BITS>;
  static constexpr int SIGHT = CODES + (BITS == 4 ? 8 : 7) * kBlock * 4, QUERIES = SIGHT + TreeRows<BITS, RB>::SIGHT * 4;
  static constexpr int BYTES = QUERIES + (RB > 1 ? RB * 4096 : 0);
};
template <int BITS, int RB, int WAVES>
constexpr int tree_lds() {
  const int merge = WAVES * 16 * (kDimRow + 2) * 4, codes = WAVES * TreeLds<BITS, RB>::BYTES;
  return merge > codes ? merge : codes;
}

template <int BITS, bool P16, int RB, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2)
attn_tree_part(const uint16_t* q, const int32_t* cu, const int32_t* lens, uint32_t magic_tiles, uint32_t magic_heads,
               uint32_t magic_group, TreeArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  using W = TreeLds<BITS, RB>;
  constexpr int ROWS = 16 * RB, ROW = BITS * 16;  // of the workgroup; bytes of a token's codes
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  TreePlace p;
  if (!find_place<ROWS>(cu, lens, magic_tiles, magic_heads, magic_group, a, p)) return;

  uint8_t* const vlds = lds + w * W::BYTES;
  float* const coef = reinterpret_cast<float*>(vlds + W::CODES);
  v8h* const qlds = reinterpret_cast<v8h*>(vlds + W::QUERIES);
  TreeRows<BITS, RB> r;
  r.init(q, magic_group, a, p, reinterpret_cast<int*>(vlds + W::SIGHT));
  if constexpr (RB > 1) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int x = 0; x < 4; ++x) qlds[(4 * rb + x) * 64 + lane] = r.qf[rb][x];
  }

  // One column of 4 bits waits for memory more than for arithmetic, so the next block's values are asked for as soon as
  // this one's lie in LDS (64 sequences' windows of 2048 tokens: 32.4 -> 31.1 us; its keys as well, in registers of
  // their own: 32.2; two columns behind 131008 tokens 200 -> 209, one of 8 bits 33.9 -> 34.1).
  constexpr bool EARLY = RB == 1 && BITS == 4;
  constexpr int KW = BITS == 4 ? 1 : 2;  // 16-byte loads of a lane's key codes
  v4u kc[4][KW], vc[4][KW];
  float4 par;
  bool par_ok;
  // tokens without a page, or past the chunk, read page 0 and have no weight
  int64_t at[4];  // first codes of the 16 tokens of group j, which lie in one page
  auto load_values = [&](int v0, int32_t entry) __attribute__((always_inline)) {
    const int t0 = p.run.position(v0);
    const int32_t mine = valid_page(a.cache, entry), safe = max(mine, 0);
    par_ok = mine >= 0 && v0 + lane < p.last;
    // load j brings group j's: values in order, four (eight) lanes a token
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      at[j] = token_slot(a.cache, __builtin_amdgcn_readlane(safe, 16 * j), p.hk, t0 + 16 * j) * ROW;
#pragma unroll
      for (int x = 0; x < KW; ++x) vc[j][x] = *reinterpret_cast<const v4u*>(a.cache.vq + at[j] + static_cast<uint32_t>(16 * lane + 1024 * x));
    }
    par = token_params<P16>(a.cache, token_slot(a.cache, safe, p.hk, t0 + lane));
  };
  auto load_keys = [&]() __attribute__((always_inline)) {  // of the same block: token i's from its byte 16 g (32 g) on
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int x = 0; x < KW; ++x)
        kc[j][x] = *reinterpret_cast<const v4u*>(a.cache.kq + at[j] + static_cast<uint32_t>(i * ROW + (BITS == 4 ? 16 : 32) * g + 16 * x));
  };

  const int step = WAVES * kBlock;
  int v0 = p.first + w * kBlock;
  int32_t entry = -1;
  if (v0 < p.last) {
    entry = entry_of(a, p, v0 + step);
    load_values(v0, entry_of(a, p, v0));
    load_keys();
  }
  // Of a SIMD's two waves the older would be served first, and the other be left alone at the end: they take turns, by
  // the place that the machine gave them (64 drafts behind 131008 tokens: 231 -> 223 us, waves alive for 92 % of the
  // cycles instead of 85).
  uint32_t turn = __builtin_amdgcn_s_getreg(4 | 0 << 6 | 3 << 11);  // bits 0 .. 3 of HW_ID: the wave's place in its SIMD
  for (; v0 < p.last; v0 += step) {
    if (turn++ & 1)
      __builtin_amdgcn_s_setprio(1);
    else
      __builtin_amdgcn_s_setprio(0);
    // codes and coefficients to LDS (this wave's own: no barrier, its LDS operations are in order)
#pragma unroll
    for (int mm = 0; mm < 4; ++mm)
#pragma unroll
      for (int x = 0; x < KW; ++x) {
        const int row = 16 * mm + (BITS == 4 ? lane >> 2 : 8 * x + (lane >> 3));
        *reinterpret_cast<v4u*>(vlds + row * kPitch<BITS> + 16 * (lane & (BITS == 4 ? 3 : 7))) = vc[mm][x];
      }
    const uint64_t there = __ballot(par_ok);
    const uint64_t odd = token_coefs(par, par_ok, a.scale_log2e, r.down, BITS == 4 && r.apart, coef);
    asm volatile("" ::: "memory");
    const bool more = v0 + step < p.last;
    if constexpr (EARLY) {
      if (more) {
        const int32_t next = entry;
        entry = entry_of(a, p, v0 + 2 * step);
        load_values(v0 + step, next);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (RB > 1) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int x = 0; x < 4; ++x) r.qf[rb][x] = qlds[(4 * rb + x) * 64 + lane];
    }
    float s[RB][16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v8h ko[4];
      key_operands<BITS>(kc[j], ko);
      r.scores(j, ko, coef, s);
      if constexpr (RB > 1 && BITS == 4) __builtin_amdgcn_sched_barrier(0);
    }
    // the next block's codes, when the registers of this one's are free
    __builtin_amdgcn_sched_barrier(0);
    if (more) {
      if constexpr (!EARLY) load_values(v0 + step, entry);
      load_keys();
      if constexpr (!EARLY) entry = entry_of(a, p, v0 + 2 * step);
    }
    r.hide(p.run.position(v0), there, odd, coef, a, p, s);
    r.move(s);
    v8h pf[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) r.weights(rb, s[rb], coef, pf[rb]);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      v8h vo[2];
      value_operands<BITS>(vlds, dt, vo);
      r.values(dt, vo, pf);
    }
    asm volatile("" ::: "memory");
  }
  __builtin_amdgcn_s_setprio(0);

  // the waves' states of 16 rows at a time meet in LDS
  float* const red = reinterpret_cast<float*>(lds);   // [wave][row][kDimRow]
  float* const red_ml = red + WAVES * 16 * kDimRow;  // [wave][row][2]
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    r.finish(rb);
    const int left = min(16, p.rows - (p.r0 + 16 * rb));  // rows of this column
    if (left <= 0) break;                                 // the workgroup leaves together
    __syncthreads();
    if (g == 0) {
      red_ml[(w * 16 + i) * 2] = r.m[rb];
      red_ml[(w * 16 + i) * 2 + 1] = r.l[rb];
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      v4f o;
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x] = __fmaf_rn(r.acc[rb][dt][x], 512.0f, r.bsum[rb]);
      *reinterpret_cast<v4f*>(red + (w * 16 + i) * kDimRow + 16 * dt + 4 * g) = o;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < left * 32; x += 64 * WAVES) {
      const int rr = x >> 5, d = 4 * (x & 31);
      float M = -INFINITY;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) M = fmaxf(M, red_ml[(v * 16 + rr) * 2]);
      float L = 0.0f;
      v4f D = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        const float f = rescale(red_ml[(v * 16 + rr) * 2], M);
        L = __fmaf_rn(red_ml[(v * 16 + rr) * 2 + 1], f, L);
        const v4f o = *reinterpret_cast<const v4f*>(red + (v * 16 + rr) * kDimRow + d);
#pragma unroll
        for (int y = 0; y < 4; ++y) D[y] = __fmaf_rn(o[y], f, D[y]);
      }
      store_row(a, p, magic_group, p.r0 + 16 * rb + rr, d, M, L, D);
    }
  }
}

// One workgroup per (row, query head) of the sequences: the states of its chunks, of which the first one has the
// number.  With one, its workgroup has written the output.
template <int J>
__global__ void __launch_bounds__(64 * J)
attn_tree_combine(const float* part, const int32_t* cu, const int32_t* lens, int64_t B, uint16_t* out, int64_t ldo, int hq, int chunks,
                  uint32_t magic_hq, int32_t rows) {
  __shared__ float red_m[J], red_l[J];
  __shared__ float2 red_d[J][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t t, h;
  div_rem(blockIdx.x, hq, magic_hq, t, h);
  const float* pr = part + static_cast<int64_t>(blockIdx.x) * chunks * kAttnPart;
  const float number = pr[2];
  if (cu) {
    const RowSeq s = find_sequence(cu, lens, B, t);
    if (s.seq < 0 || row_position(s.len, min(s.end, rows), t) < 0) return;  // left as it was: nobody wrote its states
  }
  const int n = min(static_cast<int>(number), chunks);
  if (n <= 1) return;
  float M = -INFINITY, L = 0.0f, D0 = 0.0f, D1 = 0.0f;
  constexpr int kAhead = 8;  // chunks whose loads are in flight together
  for (int c0 = w; c0 < n; c0 += J * kAhead) {
    float2 ml[kAhead], d[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {  // (past the last chunk the last again, which is dropped)
      const float* p = pr + static_cast<int64_t>(min(c0 + J * x, n - 1)) * kAttnPart;
      ml[x] = *reinterpret_cast<const float2*>(p);
      d[x] = reinterpret_cast<const float2*>(p + 4)[lane];
    }
    float top = M;
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      if (c0 + J * x >= n) {  // not by a weight of 0: its sums may be infinite
        ml[x] = make_float2(-INFINITY, 0.0f);
        d[x] = make_float2(0.0f, 0.0f);
      }
      top = fmaxf(top, ml[x].x);
    }
    const float f0 = rescale(M, top);
    L *= f0;
    D0 *= f0;
    D1 *= f0;
    M = top;
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const float f = rescale(ml[x].x, M);
      L = __fmaf_rn(ml[x].y, f, L);
      D0 = __fmaf_rn(d[x].x, f, D0);
      D1 = __fmaf_rn(d[x].y, f, D1);
    }
  }
  if constexpr (J > 1) {
    red_d[w][lane] = make_float2(D0, D1);
    if (lane == 0) {
      red_m[w] = M;
      red_l[w] = L;
    }
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int v = 0; v < J; ++v) M = fmaxf(M, red_m[v]);
    L = D0 = D1 = 0.0f;
#pragma unroll
    for (int v = 0; v < J; ++v) {
      const float f = rescale(red_m[v], M);
      const float2 d = red_d[v][lane];
      L = __fmaf_rn(red_l[v], f, L);
      D0 = __fmaf_rn(d.x, f, D0);
      D1 = __fmaf_rn(d.y, f, D1);
    }
  }
  reinterpret_cast<uint32_t*>(out + t * ldo + static_cast<int64_t>(h) * 128)[lane] =
      M == -INFINITY ? 0u : f2h2(__fdiv_rn(D0, L), __fdiv_rn(D1, L));
}

template <int BITS, bool P16, int RB, int WAVES>
hipError_t launch_part(const TreeArgs& a, hipStream_t stream) {
  constexpr auto kern = attn_tree_part<BITS, P16, RB, WAVES>;
  constexpr int lds = tree_lds<BITS, RB, WAVES>();
  const hipError_t init = set_max_lds<kern>(lds);
  if (init != hipSuccess) return init;
  const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(a.plan.tiles) * a.cache.heads * a.plan.chunks);
  return launch(kern, dim3(blocks), dim3(64 * WAVES), lds, stream, a.q, a.cu, a.lens, div_magic(static_cast<uint32_t>(a.plan.tiles)),
                div_magic(static_cast<uint32_t>(a.cache.heads)), div_magic(static_cast<uint32_t>(a.group)), a);
}

template <int RB, int WAVES>
hipError_t launch_parts(const TreeArgs& a, hipStream_t stream) {
  if (a.bits == 8) return a.param16 ? launch_part<8, true, RB, WAVES>(a, stream) : launch_part<8, false, RB, WAVES>(a, stream);
  return a.param16 ? launch_part<4, true, RB, WAVES>(a, stream) : launch_part<4, false, RB, WAVES>(a, stream);
}

}  // namespace

hipError_t launch_attn_tree(const TreeArgs& a, hipStream_t stream) {
  const hipError_t e = a.plan.rb == 2                  ? launch_parts<2, kPagedWaves>(a, stream)
                       : a.plan.waves > kPagedWaves ? launch_parts<1, 2 * kPagedWaves>(a, stream)
                                                    : launch_parts<1, kPagedWaves>(a, stream);
  if (e != hipSuccess || a.plan.chunks == 1) return e;
  const auto join = [&](auto kern, int waves) {
    return launch(kern, dim3(static_cast<unsigned>(a.T * a.hq)), dim3(64 * waves), 0, stream, a.part, a.cu, a.lens, a.B, a.out, a.ldo,
                  a.hq, a.plan.chunks, div_magic(static_cast<uint32_t>(a.hq)), static_cast<int32_t>(a.T));
  };
  return a.plan.chunks <= 8 ? join(attn_tree_combine<1>, 1) : join(attn_tree_combine<8>, 8);
}

}  // namespace sq
