// The paged cache as it is written and read back.
//
// rope_kv_write: rotary positions on queries and keys, R3 of both (Sec. 3.1), eq. 1 codes of keys
// and values into the pages.  With position p and pair frequency f_i, the pair (u, w) of dims
// becomes (u c - w s, w c + u s), c = m cos(p f_i), s = m sin(p f_i); then y = x S_128 / sqrt(128).
//   * Queries and values: four lanes (a quad) own a head vector; lane j holds the elements
//     32 k + 8 j + e, so that a 16-byte load or store of the wave covers whole 64-byte lines, and a
//     wave has 16 vectors.  Keys: eight lanes own one, so that its 64-bit values take 32 registers
//     of a lane; the wave has eight.  A wave's vectors are all queries, all keys or all values (a
//     task), and it asks for the first ones before it knows their positions.
//   * A workgroup covers a few tokens and computes their angles once for all heads: 64 lanes, one
//     frequency each, in 64 bits (p f of a far position has no fraction left in 32), reduced to
//     turns so that sin and cos see at most half a turn.  They go through LDS.
//   * Queries are rotated in 32 bits (the result is fp16).  Keys are rotated in 64: adds and fmas
//     of 64 bits issue at the 32-bit rate here, and the codes are then those of the definition
//     but for ties, not whatever the order of 32-bit sums makes of values next to a code's border.
//     Keys are rounded once to fp32, which is what eq. 1's 32-bit steps start from.
// Bound: HBM with many rows, 17034 rows of 32 + 32 heads, 8 bits, in 171 - 188 us (706 MB: 4 TB/s of
// the 5.2 that a copy reaches; the rest is the keys' 64-bit arithmetic).  With 2048 rows of 32 + 8 heads
// (44 MB in 14 - 15 us), and in a decode step (3 - 5 us), the chain of a wave: positions, angles in 64
// bits, the vectors that were asked for before them, butterflies, codes.
// kv_read: a quad per head vector takes 4 (8) code bytes per lane and 8 elements, alpha c + beta
// by one fma, R3 once more where the plain basis is asked for (S_128 / sqrt(128) is its own
// inverse), and stores fp16.  HBM bounds it: 32768 tokens of 8 heads, 4 bits, 172 MB of which four
// fifths are written, in 37 us with everything cold (4.6 TB/s) and 28 us with three inputs in turn;
// 32236 tokens of 8 heads, 8 bits, turned back, 200 MB in 44 and 36 us.
#include "paged_device.h"
#include "paged_plan.h"
#include "sq_internal.h"

namespace sq {
namespace {

constexpr int kD = 128;
constexpr double kInvSqrtD = 0.088388347648318440550;

template <typename F>
__device__ __forceinline__ void widen8(const v4u& raw, F* e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e[2 * i] = static_cast<F>(h2f(static_cast<uint16_t>(raw[i] & 0xFFFFu)));
    e[2 * i + 1] = static_cast<F>(h2f(static_cast<uint16_t>(raw[i] >> 16)));
  }
}

// How the pairs of a head vector lie in the lanes' registers.
enum RopeForm {
  kNoRope,       // rotary_dim == 0
  kHalf128,      // dims (i, i + 64): registers k and k + 2 of the same lane
  kHalf64,       // dims (i, i + 32): registers 0 and 1
  kHalfAny,      // dims (i, i + rotary_dim / 2): the partner chunk is another lane's, read again
  kInterleaved,  // dims (2 i, 2 i + 1)
};

// Turns the pairs of a vector and scales it by 1 / sqrt(128), R3's factor, which the (cos, sin) of
// tab hold already.  e: the lane's elements, N chunks of 8, chunk k being chunk(k) of the vector's
// 16; vec: the vector in memory
template <int FORM, int N, typename F, typename F2, typename C>
__device__ __forceinline__ void rotate_pairs(F (&e)[8 * N], C chunk, const F2* tab, int rotary, const uint16_t* vec) {
  if constexpr (FORM != kHalf128) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (FORM == kNoRope || 8 * chunk(k) >= rotary)
#pragma unroll
        for (int x = 0; x < 8; ++x) e[8 * k + x] *= static_cast<F>(kInvSqrtD);
  }
  auto turn = [&](int a, int b, const F2& cs) {
    const F u = e[a], w = e[b];
    e[a] = fma(u, cs.x, -(w * cs.y));
    e[b] = fma(w, cs.x, u * cs.y);
  };
  if constexpr (FORM == kHalf128) {  // chunks k and k + N / 2
#pragma unroll
    for (int k = 0; k < N / 2; ++k)
#pragma unroll
      for (int x = 0; x < 8; ++x) turn(8 * k + x, 8 * (k + N / 2) + x, tab[8 * chunk(k) + x]);
  } else if constexpr (FORM == kHalf64 && N == 4) {  // chunks 0 and 1
#pragma unroll
    for (int x = 0; x < 8; ++x) turn(x, 8 + x, tab[8 * chunk(0) + x]);
  } else if constexpr (FORM == kHalf64 || FORM == kHalfAny) {
    const int hc = rotary / 16;  // chunks of a half
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = chunk(k);
      if (c < 2 * hc) {
        const int f = c < hc ? c : c - hc;
        F p[8];
        widen8(*reinterpret_cast<const v4u*>(vec + 8 * (c < hc ? c + hc : f)), p);
        const F sign = c < hc ? F(-1) : F(1);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const F2 cs = tab[8 * f + x];
          e[8 * k + x] = fma(e[8 * k + x], cs.x, sign * (p[x] * cs.y));
        }
      }
    }
  } else if constexpr (FORM == kInterleaved) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (8 * chunk(k) < rotary)
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(8 * k + 2 * i, 8 * k + 2 * i + 1, tab[4 * chunk(k) + i]);
  }
}

template <int N, typename C>
__device__ __forceinline__ void store_half(uint16_t* v, C chunk, const float (&e)[8 * N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v4u o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = f2h2(e[8 * k + 2 * i], e[8 * k + 2 * i + 1]);
    *reinterpret_cast<v4u*>(v + 8 * chunk(k)) = o;
  }
}

// Eq. 1 of a vector in its 32-bit steps (sq_device.h), range clipped by `clip`; codes to cq, the
// pair (alpha, beta) to ab by the lane `first` (fp32, or rounded to fp16 with the codes taken from
// the rounded pair, P16).  all(v, op): op over the vector's lanes.
template <int BITS, bool P16, int N, typename C, typename R>
__device__ __forceinline__ void quantize(const float (&e)[8 * N], C chunk, R all, bool first, float clip, uint8_t* cq, void* ab) {
  constexpr float kL = BITS == 8 ? 255.0f : 15.0f;
  float mn = e[0], mx = e[0];
#pragma unroll
  for (int r = 1; r < 8 * N; ++r) {
    mn = fminf(mn, e[r]);
    mx = fmaxf(mx, e[r]);
  }
  mn = __fmul_rn(all(mn, [](float u, float v) { return fminf(u, v); }), clip);
  mx = __fmul_rn(all(mx, [](float u, float v) { return fmaxf(u, v); }), clip);
  float alpha = __fdiv_rn(__fsub_rn(mx, mn), kL), beta = mn;
  if (alpha < kMinNormal) alpha = 1.0f;
  if constexpr (P16) {
    uint16_t a16 = f2h_sat(alpha);
    if ((a16 & 0x7FFFu) == 0) a16 = 0x3C00u;  // 1.0
    const uint16_t b16 = f2h_sat(beta);
    alpha = h2f(a16);
    beta = h2f(b16);
    if (first) *static_cast<uint32_t*>(ab) = a16 | (static_cast<uint32_t>(b16) << 16);
  } else {
    if (first) *static_cast<float2*>(ab) = make_float2(alpha, beta);
  }
  const float inv = __fdiv_rn(1.0f, alpha);
  // Codes above the top appear only where the range is clipped or its parameters are rounded;
  // v_cvt_pk_u8_f32 (which rounds half to even) itself ends at 0 and 255.
  const auto store = [&](auto cc) __attribute__((always_inline)) {
    auto arg = [&](int r) {
      const float t = __fmul_rn(__fsub_rn(e[r], beta), inv);
      return decltype(cc)::value ? __builtin_amdgcn_fmed3f(t, 0.0f, kL) : t;
    };
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if constexpr (BITS == 8) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int x = 0; x < 8; ++x) w[x >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(arg(8 * k + x), x & 3, w[x >> 2]);
        *reinterpret_cast<uint2*>(cq + 8 * chunk(k)) = make_uint2(w[0], w[1]);
      } else {
        uint32_t ev = 0, od = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ev = __builtin_amdgcn_cvt_pk_u8_f32(arg(8 * k + 2 * i), i, ev);
          od = __builtin_amdgcn_cvt_pk_u8_f32(arg(8 * k + 2 * i + 1), i, od);
        }
        *reinterpret_cast<uint32_t*>(cq + 4 * chunk(k)) = ev | (od << 4);
      }
    }
  };
  if (BITS == 4 && (P16 || clip != 1.0f))
    store(std::true_type{});
  else
    store(std::false_type{});
}

// The eight lanes of a key vector: lane bits 0, 4 and 5.  Loaded chunk k is 8 k + key_lane.
__device__ __forceinline__ int key_lane(int lane) { return (lane & 1) | ((lane >> 3) & 6); }

// Unscaled 128-point transform of the eight lanes' values (register 8 k + x: dim 64 k + 8 key_lane +
// x).  The lane bits 5 and 4 are first exchanged with the register bit k, so that their butterflies
// stay in the lane; the result's register 8 k + x is dim 64 b5 + 32 b4 + 16 k + 8 b0 + x.
__device__ __forceinline__ void key_fwht(double (&e)[16], int lane) {
#pragma unroll
  for (int h = 1; h < 16; h <<= 1)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if ((r & h) == 0) {
        const double u = e[r], w = e[r + h];
        e[r] = u + w;
        e[r + h] = u - w;
      }
  const double s1 = (lane & 1) ? -1.0 : 1.0;
#pragma unroll
  for (int r = 0; r < 16; ++r) e[r] = fma(s1, e[r], quad_swap<1>(e[r]));
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    swap_halves(e[r], e[r + 8]);
    const double u = e[r], w = e[r + 8];
    e[r] = u + w;
    e[r + 8] = u - w;
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    swap_rows(e[r], e[r + 8]);
    const double u = e[r], w = e[r + 8];
    e[r] = u + w;
    e[r + 8] = u - w;
  }
}

// Where a token of the workgroup goes: place (position) and page, -1 where it has none.
struct TokenPlace {
  int64_t pos;
  int32_t page;
};

template <int BITS, bool P16, int FORM>
__global__ void __launch_bounds__(64 * kRopeWaves, 3)
rope_kv_write(const uint16_t* q, const uint16_t* k, const uint16_t* v, const int32_t* cu, const int32_t* lens,
              int64_t t_first, RopeWriteArgs a) {
  __shared__ double2 cs[kRopeTokens][64];
  __shared__ float2 csf[kRopeTokens][64];
  __shared__ TokenPlace place[kRopeTokens];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int64_t t0 = t_first + static_cast<int64_t>(blockIdx.x) * a.tokens;
  const RopeTasks tasks = rope_tasks(a.tokens, a.hq, a.cache.heads);
  enum { kQuery, kKey, kValue };

  // A lane's vector of a task: token tt of the workgroup (-1: none), head h, its row in memory, and
  // the lane's chunks of it.
  struct Item {
    int kind, tt;
    uint32_t h;
    const uint16_t* vec;
    v4u raw[4];
  };
  auto fetch = [&](int task, Item& it) __attribute__((always_inline)) {
    it.kind = task < tasks.q ? kQuery : task < tasks.q + tasks.k ? kKey : kValue;
    const int heads = it.kind == kQuery ? a.hq : a.cache.heads;
    const int x = it.kind == kQuery ? task * 16 + (lane >> 2)
                  : it.kind == kKey ? (task - tasks.q) * 8 + ((lane >> 1) & 7)
                                    : (task - tasks.q - tasks.k) * 16 + (lane >> 2);
    uint32_t tt;
    div_rem(x, heads, it.kind == kQuery ? a.magic_hq : a.magic_hkv, tt, it.h);
    it.tt = static_cast<int>(tt) < a.tokens && t0 + tt < a.T ? static_cast<int>(tt) : -1;
    const int64_t t = t0 + max(it.tt, 0);
    it.vec = (it.kind == kQuery ? q + t * a.ldq : it.kind == kKey ? k + t * a.ldk : v + t * a.ldv) + it.h * kD;
    const int first = it.kind == kKey ? key_lane(lane) : lane & 3, step = it.kind == kKey ? 8 : 4;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (c < 2 || it.kind != kKey) it.raw[c] = *reinterpret_cast<const v4u*>(it.vec + 8 * (first + step * c));
  };
  Item it, next;
  if (wave < tasks.all()) fetch(wave, it);

  // positions, pages and angles: wave w takes the tokens w, w + waves, ...
  for (int tt = wave; tt < a.tokens; tt += waves) {
    const int64_t t = t0 + tt;
    RowSeq s{-1, 0, 0, 0};
    double f = 0.0;
    int32_t depth = 0;
    if constexpr (FORM != kNoRope) {
      if (lane < a.rotary / 2) f = a.freq[lane];
      if (a.depth && t < a.T) depth = a.depth[t];
    }
    if (t < a.T) {
      if (cu)
        s = find_sequence(cu, lens, a.B, t);
      else
        s = RowSeq{static_cast<int>(t), static_cast<int>(t), static_cast<int>(t) + 1, lens[t]};
    }
    const int64_t pos = s.seq >= 0 ? row_position(s.len, s.end, t) : -1;
    int32_t entry = -1;
    const int32_t col = table_column(a.cache, pos);
    if (col >= 0) entry = a.cache.table[s.seq * a.cache.ldt + col];
    if constexpr (FORM != kNoRope) {
      // with depths, the position in the text is not the place in the cache
      const int64_t at = a.depth ? row_position(s.len, s.end, s.begin) + depth : pos;
      const double turns = static_cast<double>(at) * (f * 0.15915494309189533577);
      double sn, cn;
      sincospi(2.0 * (turns - rint(turns)), &sn, &cn);
      const double m = static_cast<double>(a.magnitude) * kInvSqrtD;
      cs[tt][lane] = make_double2(m * cn, m * sn);
      csf[tt][lane] = make_float2(static_cast<float>(m * cn), static_cast<float>(m * sn));
    }
    if (lane == 0) place[tt] = {pos, valid_page(a.cache, entry)};
  }
  __syncthreads();

  for (int task = wave; task < tasks.all(); task += waves) {
    if (task != wave) it = next;
    if (task + waves < tasks.all()) fetch(task + waves, next);  // while this one is worked on
    if (it.tt < 0) continue;  // a vector's lanes leave together
    const TokenPlace pl = place[it.tt];
    if (pl.pos < 0) continue;
    const int64_t t = t0 + it.tt;
    const int64_t slot = token_slot(a.cache, pl.page, it.h, pl.pos);
    const auto quad_chunk = [&](int c) { return 4 * c + (lane & 3); };
    const auto quad_all = [](float x, auto op) {
      x = op(x, quad_swap<1>(x));
      return op(x, quad_swap<2>(x));
    };
    if (it.kind == kKey) {
      double d[16];
#pragma unroll
      for (int c = 0; c < 2; ++c) widen8(it.raw[c], d + 8 * c);
      rotate_pairs<FORM, 2>(d, [&](int c) { return 8 * c + key_lane(lane); }, cs[it.tt], a.rotary, it.vec);
      key_fwht(d, lane);
      const auto chunk = [&](int c) { return (lane & 1) + 2 * c + ((lane >> 2) & 12); };
      float e[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) e[r] = static_cast<float>(d[r]);
      if (a.k_rot) store_half<2>(a.k_rot + (t * a.cache.heads + it.h) * kD, chunk, e);
      if (pl.page < 0) continue;
      const auto all = [](float x, auto op) { return rows_all(op(x, quad_swap<1>(x)), op); };
      void* ab = static_cast<uint8_t*>(a.cache.params) + 4 * slot * (P16 ? 2 : 4);
      quantize<BITS, P16, 2>(e, chunk, all, (lane & 49) == 0, a.k_clip, a.cache.kq + slot * (kD * BITS / 8), ab);
      continue;
    }
    float e[32];
#pragma unroll
    for (int c = 0; c < 4; ++c) widen8(it.raw[c], e + 8 * c);
    if (it.kind == kQuery) {
      rotate_pairs<FORM, 4>(e, quad_chunk, csf[it.tt], a.rotary, it.vec);
      quad_fwht(e, lane & 3);
      store_half<4>(a.q_rot + (t * a.hq + it.h) * kD, quad_chunk, e);
    } else if (pl.page >= 0) {
      void* ab = static_cast<uint8_t*>(a.cache.params) + (4 * slot + 2) * (P16 ? 2 : 4);
      quantize<BITS, P16, 4>(e, quad_chunk, quad_all, (lane & 3) == 0, a.v_clip, a.cache.vq + slot * (kD * BITS / 8), ab);
    }
  }
}

template <int BITS, bool P16, bool PLAIN>
__global__ void __launch_bounds__(256)
kv_read(const int32_t* cu, const int32_t* lens, int64_t t_first, KvReadArgs a) {
  __shared__ TokenPlace place[kReadTokens];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = lane & 3;
  const int64_t t0 = t_first + static_cast<int64_t>(blockIdx.x) * a.tokens;
  for (int tt = wave; tt < a.tokens; tt += 4) {
    const int64_t t = t0 + tt;
    RowSeq s{-1, 0, 0, 0};
    if (t < a.T) s = find_sequence(cu, lens, a.B, t);
    if (lane == 0) {
      int64_t pos = -1;
      int32_t page = -1;
      if (s.seq >= 0) pos = row_position(s.len, s.end, t);
      if (pos >= 0) {
        const int32_t col = table_column(a.cache, pos);
        if (col >= 0) page = valid_page(a.cache, a.cache.table[s.seq * a.cache.ldt + col]);
      }
      place[tt] = {pos, page};
    }
  }
  __syncthreads();
  for (int x = threadIdx.x / 4; x < a.tokens * a.cache.heads; x += 64) {
    uint32_t tt, h;
    div_rem(x, a.cache.heads, a.magic_hkv, tt, h);
    const int64_t t = t0 + tt;
    const TokenPlace pl = place[tt];
    if (t >= a.T || pl.pos < 0) continue;  // the quad's lanes leave together
    float e[2][32];
    if (pl.page >= 0) {
      const int64_t slot = token_slot(a.cache, pl.page, h, pl.pos);
      float ab[4];
      if constexpr (P16) {
        const uint2 p = static_cast<const uint2*>(a.cache.params)[slot];
        ab[0] = h2f(static_cast<uint16_t>(p.x));
        ab[1] = h2f(static_cast<uint16_t>(p.x >> 16));
        ab[2] = h2f(static_cast<uint16_t>(p.y));
        ab[3] = h2f(static_cast<uint16_t>(p.y >> 16));
      } else {
        const float4 p = static_cast<const float4*>(a.cache.params)[slot];
        ab[0] = p.x, ab[1] = p.y, ab[2] = p.z, ab[3] = p.w;
      }
      if constexpr (PLAIN) {
        ab[0] = __fmul_rn(ab[0], static_cast<float>(kInvSqrtD));
        ab[1] = __fmul_rn(ab[1], static_cast<float>(kInvSqrtD));
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint8_t* codes = (s ? a.cache.vq : a.cache.kq) + slot * (kD * BITS / 8);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (BITS == 8) {
            const uint2 w = *reinterpret_cast<const uint2*>(codes + 32 * k + 8 * j);
#pragma unroll
            for (int y = 0; y < 8; ++y)
              e[s][8 * k + y] = __fmaf_rn(static_cast<float>(((y < 4 ? w.x : w.y) >> (8 * (y & 3))) & 0xFFu), ab[2 * s], ab[2 * s + 1]);
          } else {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + 16 * k + 4 * j);
#pragma unroll
            for (int y = 0; y < 8; ++y)
              e[s][8 * k + y] = __fmaf_rn(static_cast<float>((w >> (4 * y)) & 0xFu), ab[2 * s], ab[2 * s + 1]);
          }
        }
      }
    } else {  // a page that is not in the pool reads as zeros
#pragma unroll
      for (int r = 0; r < 32; ++r) e[0][r] = e[1][r] = 0.0f;
    }
    if constexpr (PLAIN) quad_fwht(e[0], j);  // its 1 / sqrt(128) is in the parameters
    const auto chunk = [&](int c) { return 4 * c + j; };
    store_half<4>(a.k + t * a.ldk + h * kD, chunk, e[0]);
    store_half<4>(a.v + t * a.ldv + h * kD, chunk, e[1]);
  }
}

}  // namespace

hipError_t launch_rope_kv_write(RopeWriteArgs a, hipStream_t stream) {
  const RopePlan plan = rope_plan(a.T, a.hq, a.cache.heads);
  const int tokens = plan.tokens, threads = 64 * plan.waves;
  a.tokens = tokens;
  a.magic_hq = div_magic(static_cast<uint32_t>(a.hq));
  a.magic_hkv = div_magic(static_cast<uint32_t>(a.cache.heads));
  const int form = a.rotary == 0     ? kNoRope
                   : a.interleaved   ? kInterleaved
                   : a.rotary == 128 ? kHalf128
                   : a.rotary == 64  ? kHalf64
                                     : kHalfAny;
  return in_parts(a.T, max_blocks(threads) * tokens, [&](int64_t t, int64_t n) {
    const dim3 grid(static_cast<unsigned>((n + tokens - 1) / tokens));
    hipError_t e = hipErrorInvalidValue;
    static_for<5>([&](auto fc) {
      constexpr int F = decltype(fc)::value;
      if (form != F) return;
      const auto go = [&](auto kern) { e = launch(kern, grid, dim3(threads), 0, stream, a.q, a.k, a.v, a.cu, a.lens, t, a); };
      if (a.bits == 8)
        a.param16 ? go(rope_kv_write<8, true, F>) : go(rope_kv_write<8, false, F>);
      else
        a.param16 ? go(rope_kv_write<4, true, F>) : go(rope_kv_write<4, false, F>);
    });
    return e;
  });
}

hipError_t launch_kv_read(KvReadArgs a, hipStream_t stream) {
  int tokens = 64 / a.cache.heads;  // one vector pair per quad of the workgroup's 64
  tokens = tokens < 1 ? 1 : tokens > kReadTokens ? kReadTokens : tokens;
  a.tokens = tokens;
  a.magic_hkv = div_magic(static_cast<uint32_t>(a.cache.heads));
  return in_parts(a.T, max_blocks(256) * tokens, [&](int64_t t, int64_t n) {
    const dim3 grid(static_cast<unsigned>((n + tokens - 1) / tokens));
    const auto go = [&](auto kern) { return launch(kern, grid, dim3(256), 0, stream, a.cu, a.lens, t, a); };
    const auto pick = [&](auto plain) {
      constexpr bool P = decltype(plain)::value;
      if (a.bits == 8) return a.param16 ? go(kv_read<8, true, P>) : go(kv_read<8, false, P>);
      return a.param16 ? go(kv_read<4, true, P>) : go(kv_read<4, false, P>);
    };
    return a.plain_basis ? pick(std::true_type{}) : pick(std::false_type{});
  });
}

}  // namespace sq
