// The paged cache as it is written and read back.
//
// rope_kv_write: rotary positions on queries and keys, R3 of both (Sec. 3.1), eq. 1 codes of keys
// and values into the pages.  With position p and pair frequency f_i, the pair (u, w) of dims
// becomes (u c - w s, w c + u s), c = m cos(p f_i), s = m sin(p f_i); then y = x S_128 / sqrt(128).
//   * Four lanes (a quad) own a head vector; lane j holds the elements 32 k + 8 j + e, so that a
//     16-byte load or store of the wave covers whole 64-byte lines.  A wave's 16 vectors are all
//     queries, all keys or all values (a `task`): keys cost three times a query.
//   * A workgroup covers TB tokens and computes their angles once for all heads: 64 lanes, one
//     frequency each, in 64 bits (p f of a far position has no fraction left in 32), reduced to
//     turns so that sin and cos see at most half a turn.  They go through LDS.
//   * Queries are rotated in 32 bits (the result is fp16).  Keys are rotated in 64: adds and fmas
//     of 64 bits issue at the 32-bit rate here, and the codes are then those of the definition
//     but for ties, not whatever the order of 32-bit sums makes of values next to a code's border.
//     Keys are rounded once to fp32, which is what eq. 1's 32-bit steps start from.
// kv_read: a quad per head vector takes 4 (8) code bytes per lane and 8 elements, alpha c + beta
// by one fma, R3 once more where the plain basis is asked for (S_128 / sqrt(128) is its own
// inverse), and stores fp16.
#include "paged_device.h"
#include "sq_internal.h"

namespace sq {
namespace {

constexpr int kD = 128;
constexpr float kInvSqrtD = 0.08838834764831845f;

// the lane's four 16-byte chunks of a head vector: chunk k holds elements 32 k + 8 j .. + 7
__device__ __forceinline__ void load_chunks(const uint16_t* v, int j, v4u (&raw)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) raw[k] = *reinterpret_cast<const v4u*>(v + 32 * k + 8 * j);
}
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

// e: the lane's elements; tab: (cos, sin) per frequency; vec: the vector in memory
template <int FORM, typename F, typename F2>
__device__ __forceinline__ void rotate_pairs(F (&e)[32], int j, const F2* tab, int rotary, const uint16_t* vec) {
  auto turn = [&](int a, int b, const F2& cs) {
    const F u = e[a], w = e[b];
    e[a] = fma(u, cs.x, -(w * cs.y));
    e[b] = fma(w, cs.x, u * cs.y);
  };
  if constexpr (FORM == kHalf128) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int x = 0; x < 8; ++x) turn(8 * k + x, 8 * (k + 2) + x, tab[8 * (4 * k + j) + x]);
  } else if constexpr (FORM == kHalf64) {
#pragma unroll
    for (int x = 0; x < 8; ++x) turn(x, 8 + x, tab[8 * j + x]);
  } else if constexpr (FORM == kHalfAny) {
    const int hc = rotary / 16;  // chunks of a half
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = 4 * k + j;
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
    for (int k = 0; k < 4; ++k)
      if (8 * (4 * k + j) < rotary)
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(8 * k + 2 * i, 8 * k + 2 * i + 1, tab[4 * (4 * k + j) + i]);
  }
}

__device__ __forceinline__ void store_half(uint16_t* v, int j, const float (&e)[32], float scale) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v4u o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = f2h2(__fmul_rn(e[8 * k + 2 * i], scale), __fmul_rn(e[8 * k + 2 * i + 1], scale));
    *reinterpret_cast<v4u*>(v + 32 * k + 8 * j) = o;
  }
}

// Eq. 1 of the quad's vector in its 32-bit steps (sq_device.h), range clipped by `clip`; codes to
// cq, the pair (alpha, beta) to ab (fp32, or rounded to fp16 with the codes taken from the rounded
// pair, P16).
template <int BITS, bool P16>
__device__ __forceinline__ void quantize(const float (&e)[32], int j, float clip, uint8_t* cq, void* ab) {
  constexpr float kL = BITS == 8 ? 255.0f : 15.0f;
  float mn = e[0], mx = e[0];
#pragma unroll
  for (int r = 1; r < 32; ++r) {
    mn = fminf(mn, e[r]);
    mx = fmaxf(mx, e[r]);
  }
  mn = fminf(mn, quad_swap<1>(mn));
  mx = fmaxf(mx, quad_swap<1>(mx));
  mn = __fmul_rn(fminf(mn, quad_swap<2>(mn)), clip);
  mx = __fmul_rn(fmaxf(mx, quad_swap<2>(mx)), clip);
  float alpha = __fdiv_rn(__fsub_rn(mx, mn), kL), beta = mn;
  if (alpha < kMinNormal) alpha = 1.0f;
  if constexpr (P16) {
    uint16_t a16 = f2h_sat(alpha);
    if ((a16 & 0x7FFFu) == 0) a16 = 0x3C00u;  // 1.0
    const uint16_t b16 = f2h_sat(beta);
    alpha = h2f(a16);
    beta = h2f(b16);
    if (j == 0) *static_cast<uint32_t*>(ab) = a16 | (static_cast<uint32_t>(b16) << 16);
  } else {
    if (j == 0) *static_cast<float2*>(ab) = make_float2(alpha, beta);
  }
  const float inv = __fdiv_rn(1.0f, alpha);
  auto arg = [&](int r) { return __builtin_amdgcn_fmed3f(__fmul_rn(__fsub_rn(e[r], beta), inv), 0.0f, kL); };
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (BITS == 8) {
      uint32_t w[2] = {0u, 0u};
#pragma unroll
      for (int x = 0; x < 8; ++x) w[x >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(arg(8 * k + x), x & 3, w[x >> 2]);
      *reinterpret_cast<uint2*>(cq + 32 * k + 8 * j) = make_uint2(w[0], w[1]);
    } else {
      uint32_t ev = 0, od = 0;  // v_cvt_pk_u8_f32 rounds half to even
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ev = __builtin_amdgcn_cvt_pk_u8_f32(arg(8 * k + 2 * i), i, ev);
        od = __builtin_amdgcn_cvt_pk_u8_f32(arg(8 * k + 2 * i + 1), i, od);
      }
      *reinterpret_cast<uint32_t*>(cq + 16 * k + 4 * j) = ev | (od << 4);
    }
  }
}

// Where a token of the workgroup goes: place (position) and page, -1 where it has none.
struct TokenPlace {
  int64_t pos;
  int32_t page;
};

template <int BITS, bool P16, int FORM>
__global__ void __launch_bounds__(1024)
rope_kv_write(const uint16_t* q, const uint16_t* k, const uint16_t* v, const int32_t* cu, const int32_t* lens,
              int64_t t_first, RopeWriteArgs a) {
  __shared__ double2 cs[kRopeTokens][64];
  __shared__ float2 csf[kRopeTokens][64];
  __shared__ TokenPlace place[kRopeTokens];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int j = lane & 3;
  const int64_t t0 = t_first + static_cast<int64_t>(blockIdx.x) * a.tokens;
  const int nq = (a.tokens * a.hq + 15) / 16, nk = (a.tokens * a.cache.heads + 15) / 16;

  // positions, pages and angles: wave w takes the tokens w, w + waves, ...
  for (int tt = wave; tt < a.tokens; tt += waves) {
    const int64_t t = t0 + tt;
    RowSeq s{-1, 0, 0};
    if (t < a.T) {
      if (cu)
        s = find_sequence(cu, a.B, t);
      else
        s = RowSeq{static_cast<int>(t), static_cast<int>(t), static_cast<int>(t) + 1};
    }
    int64_t pos = -1;
    if (s.seq >= 0) pos = row_position(lens[s.seq], s.end, t);
    if constexpr (FORM != kNoRope) {
      if (lane < a.rotary / 2) {
        const double turns = static_cast<double>(pos) * (a.freq[lane] * 0.15915494309189533577);
        double sn, cn;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cn);
        const double m = static_cast<double>(a.magnitude);
        cs[tt][lane] = make_double2(m * cn, m * sn);
        csf[tt][lane] = make_float2(static_cast<float>(m * cn), static_cast<float>(m * sn));
      }
    }
    if (lane == 0) {
      int32_t page = -1;
      if (pos >= 0) {
        const int32_t col = table_column(a.cache, pos);
        if (col >= 0) page = valid_page(a.cache, a.cache.table[s.seq * a.cache.ldt + col]);
      }
      place[tt] = {pos, page};
    }
  }
  __syncthreads();

  for (int task = wave; task < nq + 2 * nk; task += waves) {
    const int kind = task < nq ? 0 : task < nq + nk ? 1 : 2;  // queries, keys, values
    const int heads = kind == 0 ? a.hq : a.cache.heads;
    uint32_t tt, h;
    div_rem((task - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * 16 + lane / 4, heads, kind == 0 ? a.magic_hq : a.magic_hkv,
            tt, h);
    if (static_cast<int>(tt) >= a.tokens || t0 + tt >= a.T) continue;  // the quad's lanes leave together
    const TokenPlace pl = place[tt];
    if (pl.pos < 0) continue;
    const int64_t t = t0 + tt;
    const uint16_t* vec = (kind == 0 ? q + t * a.ldq : kind == 1 ? k + t * a.ldk : v + t * a.ldv) + h * kD;
    const int64_t slot = pl.page >= 0 ? token_slot(a.cache, pl.page, h, pl.pos) : -1;
    v4u raw[4];
    load_chunks(vec, j, raw);
    float e[32];
    if (kind == 0) {
#pragma unroll
      for (int c = 0; c < 4; ++c) widen8(raw[c], e + 8 * c);
      rotate_pairs<FORM>(e, j, csf[tt], a.rotary, vec);
      quad_fwht(e, j);
      store_half(a.q_rot + (t * a.hq + h) * kD, j, e, kInvSqrtD);
      continue;
    }
    if (kind == 1) {
      double d[32];
#pragma unroll
      for (int c = 0; c < 4; ++c) widen8(raw[c], d + 8 * c);
      rotate_pairs<FORM>(d, j, cs[tt], a.rotary, vec);
      quad_fwht(d, j);
#pragma unroll
      for (int r = 0; r < 32; ++r) e[r] = static_cast<float>(d[r] * 0.088388347648318440550);
      if (a.k_rot) store_half(a.k_rot + (t * a.cache.heads + h) * kD, j, e, 1.0f);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) widen8(raw[c], e + 8 * c);
    }
    if (slot < 0) continue;
    uint8_t* codes = (kind == 1 ? a.cache.kq : a.cache.vq) + slot * (kD * BITS / 8);
    void* ab = static_cast<uint8_t*>(a.cache.params) + (4 * slot + 2 * (kind - 1)) * (P16 ? 2 : 4);
    quantize<BITS, P16>(e, j, kind == 1 ? a.k_clip : a.v_clip, codes, ab);
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
    RowSeq s{-1, 0, 0};
    if (t < a.T) s = find_sequence(cu, a.B, t);
    if (lane == 0) {
      int64_t pos = -1;
      int32_t page = -1;
      if (s.seq >= 0) pos = row_position(lens[s.seq], s.end, t);
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
    if constexpr (PLAIN) quad_fwht(e[0], j);
    store_half(a.k + t * a.ldk + h * kD, j, e[0], PLAIN ? kInvSqrtD : 1.0f);
    store_half(a.v + t * a.ldv + h * kD, j, e[1], 1.0f);
  }
}

}  // namespace

hipError_t launch_rope_kv_write(RopeWriteArgs a, hipStream_t stream) {
  // Tokens of a workgroup: as many as give each of its (at most 16) waves one task of 16 vectors.
  int tokens = 1;
  const auto tasks_of = [&](int n) { return (n * a.hq + 15) / 16 + 2 * ((n * a.cache.heads + 15) / 16); };
  while (tokens < kRopeTokens && tokens < a.T && tasks_of(2 * tokens) <= 16) tokens *= 2;
  a.tokens = tokens;
  const int tasks = tasks_of(tokens);
  const int threads = 64 * (tasks < 16 ? tasks : 16);
  a.magic_hq = div_magic(static_cast<uint32_t>(a.hq));
  a.magic_hkv = div_magic(static_cast<uint32_t>(a.cache.heads));
  const int form = a.rotary == 0 ? kNoRope : a.interleaved ? kInterleaved : a.rotary == 128 ? kHalf128 : a.rotary == 64 ? kHalf64 : kHalfAny;
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
