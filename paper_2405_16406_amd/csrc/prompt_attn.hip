// Causal attention of packed sequences in fp16 with shared key/value heads (a whole prompt, or a
// chunk whose keys began earlier):
//     out = softmax_t(scale q_i . k_t) V over t <= m - n + i (causal), n rows and m keys of the
//     sequence; a row that sees nothing is zero.
//
// A workgroup of eight waves serves one (sequence, key/value head) and 256 of its rows, a row
// being a (token, query head of the group) pair, heads fastest: the heads that share keys share
// the tile, and a group's few tokens fill it as well as one head's many.  A wave owns 32 rows and
// walks the keys in tiles of 64:
//   scores   S^T = K Q^T by 32x32x16 products.  A lane then holds 32 of a tile's 64 scores of ONE
//            row (lane % 32), so the softmax's maximum and sum are in the lane but for one
//            exchange of the wave's halves, and its factors are one value a lane.
//   softmax  in base 2 and fp32: weights 2^(s - m), their sum l, m kWeightBits below the running
//            maximum.  m moves, and the output is rescaled, only where the largest weight would grow
//            by more than 2^kSlack.
//   values   O^T += V^T P^T.  The slots of the product's inner index may hold the keys in any
//            order, the same for both operands: in the order in which the first product leaves
//            the scores, the rounded weights are an operand as they are; V comes from LDS by
//            transposed reads (ds_read_b64_tr_b16) of the same keys.
// Tiles of K and V go from memory straight to LDS, one ahead of the products.  A tile's row is 256
// bytes; its 16-byte chunk c lies at c xor swizzle(row), so that neither the 16 rows of a K read
// nor the 4 x 64 bytes of a transposed read of V meet on a bank.
// Weights are rounded to fp16, as the second product needs them: 2^-12 of a weight down to 2^-14, where
// the largest is 2^7 to 2^15, and 2^-25 below.  Sums stay in fp32.  Outputs are off by 2.5e-4 to 2.9e-4
// of their size, of which the output's own rounding is 2.0e-4.
// The matrix cores bound it where there are rows and keys enough: 2048 tokens behind 32768 (64
// heads on 8) take 1950 us, 1.16 PFLOP/s, the rate a large library product reaches on the card.  They
// are busy for 68 % of the cycles, at 1.53 - 1.57 GHz: the chip's power sets the clock.  LDS is at 34 %,
// without bank conflicts.
// Shorter prompts add what a workgroup does once (find the tile, first keys and queries, first scores
// and last values alone, stores) and what a causal prompt's last tile wastes: one of a single tile
// takes 7 us, and a tile of a long one 1.8.  16 packed prompts of 292 .. 4000 tokens, 32 heads on 8,
// 431 - 439 us (0.9 PFLOP/s, matrix cores busy for 44 - 46 % at 1.7 GHz), 2048 tokens of 32 heads 49 - 51
// us (0.7).  Two workgroups of four waves a compute unit, each with its own keys, would hide one's
// start behind the other's products: 51 - 52, 442 and 2020 - 2040 us for these three, no gain.
//
// Few rows over many keys (a follow-up question on a long document) would leave most of the chip
// idle: the keys are then split over workgroups, whose fp32 states a second kernel joins.
#include "paged_device.h"
#include "paged_plan.h"
#include "sq_internal.h"

namespace sq {
namespace {

constexpr int kWaves = 8;
constexpr int kTile = kPromptTile;          // keys of a tile
constexpr int kTileBytes = kTile * 256;     // of K, and of V
constexpr float kSlack = 8.0f;              // log2: weights stay below 2^(kWeightBits + kSlack) < 65504
constexpr float kWeightBits = 7.0f;         // the largest weight when m has just moved
// Scores of this size have steps of 1/2.  From there on m is the maximum itself, since kWeightBits below
// it might be rounded to more than fp16 holds, and a weight is that of the rounded score, not of the
// exact product with the scale, which may be far above the rounded maximum: both gave NaN.
constexpr float kLargeScore = 4194304.0f;   // 2^22

// KG groups of waves share a workgroup's rows and take its tiles of keys in turn.
template <int KG>
struct Prompt {
  static constexpr int ROWS = 32 * kWaves / KG;   // of the workgroup, 32 of a wave
  static constexpr int LDS = KG * 4 * kTileBytes;  // two tiles of K and of V for each group
  static constexpr int COPIES = 2 * KG;            // 1 KB copies of a wave for a tile of K, or V
};

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

// where the 16-byte chunks of row t of a tile lie: c -> c ^ swizzle(t)
__device__ __forceinline__ int swizzle(int t) { return ((t & 3) << 2) | ((t >> 2) & 3); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rescale(float a, float b) { return a == -INFINITY ? 0.0f : exp2_fast(__fsub_rn(a, b)); }

// op over the lane's value and that of the other half of the wave
template <typename Op>
__device__ __forceinline__ float halves(float v, Op op) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// Schedule of a run of N products whose first operand takes R LDS reads: reads stay AHEAD operands
// in front (the compiler would read all of them first and run out of registers).
template <int N, int R, int AHEAD>
__device__ __forceinline__ void pace() {
  __builtin_amdgcn_sched_group_barrier(0x100, R * AHEAD, 0);  // LDS reads
  static_for<N - AHEAD>([](auto) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  });
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// Inclusive sum over the lanes of a wave up to each: rows of 16 by shifts, then the rows' totals.
__device__ __forceinline__ int wave_scan(int v) {
  const auto add = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  };
  using std::integral_constant;
  add(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});  // row_shr:1
  add(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});  // row_bcast:15
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});  // row_bcast:31
  return v;
}

// Sequence and tile of the tile number `rem` among ceil(rows / ROWS) tiles a sequence.
struct PromptTile {
  int seq;          // -1: past the last
  int tile, tiles;
  int q0, n;        // first row of q and rows of the sequence
  int k0, m;        // first row of k and its keys
};
template <int ROWS>
__device__ __forceinline__ PromptTile find_tile(const int32_t* cu_q, const int32_t* cu_k, int64_t B, int64_t Tq, int64_t Tk, int group,
                                                int rem) {
  const int lane = threadIdx.x & 63;
  for (int64_t b0 = 0; b0 < B; b0 += 64) {
    int q0 = 0, n = 0, k0 = 0, m = 0;
    if (b0 + lane < B) {  // clamped to the tensors, whatever cu_q and cu_k hold
      const int lq = static_cast<int>(Tq), lk = static_cast<int>(Tk);
      const int a = cu_q[b0 + lane], b = cu_q[b0 + lane + 1], c = cu_k[b0 + lane], d = cu_k[b0 + lane + 1];
      q0 = min(max(a, 0), lq);
      n = max(min(b, lq) - q0, 0);
      k0 = min(max(c, 0), lk);
      m = max(min(d, lk) - k0, 0);
    }
    const int tiles = (n * group + ROWS - 1) / ROWS;
    const int upto = wave_scan(tiles);
    const uint64_t past = __ballot(upto > rem);
    if (past) {
      const int f = __builtin_ctzll(past);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
      return {static_cast<int>(b0) + f, rem - (of(upto) - of(tiles)), of(tiles), of(q0), of(n), of(k0), of(m)};
    }
    rem -= __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, 0, 0, 0, 0, 0};
}

template <bool SPLIT, int KG>
__global__ void __launch_bounds__(64 * kWaves, 2)
attn_prompt_tile(const uint16_t* q, const uint16_t* k, const uint16_t* v, const int32_t* cu_q, const int32_t* cu_k,
                 uint32_t magic_heads, uint32_t magic_group, uint32_t magic_splits, PromptArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  using P = Prompt<KG>;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int late = w >> 2;              // the second of a SIMD's two waves
  const int rw = KG == 1 ? w : w & 3;   // which rows,
  const int kg = KG == 1 ? 0 : late;    // and which group of waves
  const int col = lane & 31, h = lane >> 5;
  uint32_t rest, hk, split = 0;
  div_rem(blockIdx.x, a.hkv, magic_heads, rest, hk);
  if constexpr (SPLIT) {
    uint32_t r2;
    div_rem(rest, a.splits, magic_splits, r2, split);
    rest = r2;
  }
  const PromptTile pt = find_tile<P::ROWS>(cu_q, cu_k, a.B, a.Tq, a.Tk, a.group, static_cast<int>(rest));
  if (pt.seq < 0) return;  // the workgroup leaves together
  const int tile = a.causal ? pt.tiles - 1 - pt.tile : pt.tile;  // the longest first
  const int k0 = pt.k0, m = pt.m;
  const int rows = pt.n * a.group;

  // this lane's row: rows past the last repeat it and are not stored
  const int row = tile * P::ROWS + 32 * rw + col;
  uint32_t tok, gh;
  div_rem(static_cast<uint32_t>(min(row, rows - 1)), a.group, magic_group, tok, gh);
  const int64_t head = static_cast<int64_t>(hk) * a.group + gh;
  const int64_t qrow = pt.q0 + static_cast<int64_t>(tok);
  // last key this row sees; of the wave's first and last rows and of the workgroup's last
  const auto limit = [&](int r) {
    if (!a.causal) return m - 1;
    uint32_t t, x;
    div_rem(static_cast<uint32_t>(min(r, rows - 1)), a.group, magic_group, t, x);
    return min(m - pt.n + static_cast<int>(t), m - 1);
  };
  const int lim = limit(row);
  const int wave_lo = limit(tile * P::ROWS + 32 * rw), wave_hi = limit(tile * P::ROWS + 32 * rw + 31);
  const int keys = limit(tile * P::ROWS + P::ROWS - 1) + 1;  // of the workgroup
  const int tiles_all = keys > 0 ? (keys + kTile - 1) / kTile : 0;
  int kt0 = 0, kt1 = tiles_all;
  if constexpr (SPLIT) {
    const int per = prompt_part(tiles_all, a.splits, a.per);
    kt0 = min(static_cast<int>(split) * per, tiles_all);
    kt1 = min(kt0 + per, tiles_all);
    if (split > 0 && kt0 == kt1) return;  // the workgroup leaves together; part 0 is always there
  }

  // Q^T operands: lane (row, h) holds dims 16 s + 8 h .. + 7
  v8h qf[8];
  {
    const uint16_t* qp = q + qrow * a.ldq + head * 128 + 8 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const v8h*>(qp + 16 * s);
  }

  // copies: copy x of a tile brings rows 4 x .. 4 x + 3; wave rw of the group takes COPIES of them
  const int ldk2 = static_cast<int>(a.ldk * 2), ldv2 = static_cast<int>(a.ldv * 2);
  int koff[P::COPIES], voff[P::COPIES];
#pragma unroll
  for (int x = 0; x < P::COPIES; ++x) {
    const int r = 4 * (P::COPIES * rw + x) + (lane >> 4);
    const int c = (lane & 15) ^ swizzle(r);
    koff[x] = r * ldk2 + 16 * c;
    voff[x] = r * ldv2 + 16 * c;
  }
  const uint8_t* const kbase = reinterpret_cast<const uint8_t*>(k + k0 * a.ldk + static_cast<int64_t>(hk) * 128);
  const uint8_t* const vbase = reinterpret_cast<const uint8_t*>(v + k0 * a.ldv + static_cast<int64_t>(hk) * 128);
  typedef __attribute__((address_space(3))) void* lds_ptr;
  auto issue = [&](int kt, int buf, bool keys_of) __attribute__((always_inline)) {
    // rows past the last key are out of the buffer and land as zeros
    const int rows_here = min(kTile, m - kt * kTile), ld2 = keys_of ? ldk2 : ldv2;
    const __amdgpu_buffer_rsrc_t rs =
        buf_rsrc((keys_of ? kbase : vbase) + static_cast<int64_t>(kt) * kTile * ld2, static_cast<int64_t>(rows_here - 1) * ld2 + 256);
#pragma unroll
    for (int x = 0; x < P::COPIES; ++x) {
      uint8_t* dst = lds + (4 * kg + buf + (keys_of ? 0 : 2)) * kTileBytes + (P::COPIES * rw + x) * 1024;
      const int off = keys_of ? koff[x] : voff[x];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(uintptr_t)dst, 16, off, 0, 0, 0);
    }
  };

  // LDS reads: K row `col` of each half tile, chunk 2 s + h; V: lane (i, gi) of 16 reads 8 bytes of
  // row 4 h + i / 4 (+ 8), dims 32 dt + 16 (gi % 2) + 4 (i % 4) .. and gets dim 32 dt + col of four
  // keys.  The lane's 16 addresses stay in registers; buffer, half tile and key step are offsets of
  // the instructions.
  uint32_t kadr[8], vadr[4][2];
#pragma unroll
  for (int x = 0; x < 8; ++x) kadr[x] = 4 * kg * kTileBytes + col * 256 + 16 * ((2 * x + h) ^ swizzle(col));
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int second = 0; second < 2; ++second) {
      const int t = 4 * h + ((lane & 15) >> 2) + 8 * second;
      const int c = 4 * dt + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
      vadr[dt][second] = 4 * kg * kTileBytes + t * 256 + 16 * (c ^ swizzle(t)) + 8 * (lane & 1);
    }
#pragma unroll
  for (int x = 0; x < 8; ++x) asm("" : "+v"(kadr[x]), "+v"(vadr[x >> 1][x & 1]));  // not derived from each other
  typedef __attribute__((address_space(3))) uint8_t* lds_bytes;
  const lds_bytes lds3 = (lds_bytes)(uintptr_t)lds;
  auto k_operand = [&](int buf, int mt, int x) __attribute__((always_inline)) -> v8h {
    return *(__attribute__((address_space(3))) const v8h*)(lds3 + kadr[x] + (buf * kTileBytes + mt * 32 * 256));
  };
  auto v_operand = [&](int buf, int ks, int dt) __attribute__((always_inline)) -> v8h {
    v4s x[2];
#pragma unroll
    for (int second = 0; second < 2; ++second)
      x[second] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) v4s*)(lds3 + vadr[dt][second] + ((2 + buf) * kTileBytes + ks * 16 * 256)));
    return __builtin_bit_cast(v8h, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };

  float mx = -INFINITY, l = 0.0f;
  v16f acc[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[dt][r] = 0.0f;
  const float cs = a.scale_log2e;
  bool large = false;  // a row of the wave has m beyond kLargeScore
  v16f s[2];   // scores of a tile: keys 32 mt + 8 (r / 4) + 4 h + r % 4
  v8h pf[4];   // its weights, an operand of the second product

  auto scores = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = 0.0f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_operand(buf, mt, x), qf[x], s[mt], 0, 0, 0);
      }
    }
    pace<16, 1, 4>();
  };

  // MASK: the tile holds keys that a row of the wave does not see
  auto softmax = [&](int kt, auto mc) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mc)::value;
    if constexpr (MASK) {
      const int left = lim - kt * kTile - 4 * h;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * mt + 8 * (r >> 2) + (r & 3) > left) s[mt][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[0][r]);
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[1][r]);
    top = halves(top, [](float x, float y) { return fmaxf(x, y); }) * cs;
    if (__builtin_expect(__ballot(top - mx > kWeightBits + kSlack) != 0, 0)) {  // (mx = -inf: any score)
      const float mn = fmaxf(mx, fabsf(top) < kLargeScore ? top - kWeightBits : top);
      const float f = rescale(mx, mn);
      l *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) acc[dt] *= f;
      mx = mn;
      large = __ballot(fabsf(mx) >= kLargeScore && mx != -INFINITY) != 0;
    }
    const float base = mx == -INFINITY ? 0.0f : mx;
    float cw = cs;
    if (__builtin_expect(large, 0)) {
#pragma unroll
      for (int r = 0; r < 32; ++r) s[r >> 4][r & 15] *= cs;
      cw = 1.0f;
    }
    // the sum is that of the rounded weights: their rounding then moves the mean of the values
    // seen, not its size
    float l0 = 0.0f, l1 = 0.0f;
    const v2h ones = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      uint32_t p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = exp2_fast(__fmaf_rn(s[ks >> 1][8 * (ks & 1) + 2 * r], cw, -base));
        const float y = exp2_fast(__fmaf_rn(s[ks >> 1][8 * (ks & 1) + 2 * r + 1], cw, -base));
        p[r] = f2h2(x, y);
        float& lr = r & 1 ? l1 : l0;
        lr = __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, p[r]), ones, lr, false);
      }
      pf[ks] = __builtin_bit_cast(v8h, v4u{p[0], p[1], p[2], p[3]});
    }
    l += l0 + l1;
    // done here: not beside the products of the next phase, which belong to the other wave's softmax
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(pf[ks]));
    asm volatile("" : "+v"(l));
  };

  // A weight of 0 does not hide a value that is not finite, and in a masked tile some rows must not
  // see what others do: there, such values stay out of the product, and what a row sees of them is
  // kept as a bit for each of the lane's 64 dims (4 y + e of chunk y): +inf, -inf, or both for NaN.
  uint64_t up = 0, down = 0;
  auto add_odd = [&](int kt, int buf) __attribute__((always_inline)) {
#pragma unroll 1
    for (int t = 0; t < kTile; ++t) {
      if (kt * kTile + t > lim) continue;
#pragma unroll 1
      for (int c = 0; c < 16; ++c) {
        const v2u u = *reinterpret_cast<const v2u*>(lds + (4 * kg + 2 + buf) * kTileBytes + t * 256 + 16 * (c ^ swizzle(t)) + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = (u[e >> 1] >> (16 * (e & 1))) & 0xFFFFu;
          if ((x & 0x7C00u) != 0x7C00u) continue;
          const uint64_t bit = uint64_t{1} << (4 * c + e);
          const bool nan = (x & 0x3FFu) != 0;
          if (nan || !(x & 0x8000u)) up |= bit;
          if (nan || (x & 0x8000u)) down |= bit;
        }
      }
    }
  };
  auto values = [&](int kt, int buf, auto mc) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mc)::value;
    if constexpr (MASK) {
      uint32_t any = 0;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          const v4u u = __builtin_bit_cast(v4u, v_operand(buf, ks, dt));
#pragma unroll
          for (int y = 0; y < 4; ++y) any |= (u[y] & 0x7C007C00u) + 0x04000400u;
        }
      pace<16, 2, 4>();
      if (__builtin_expect(__ballot((any & 0x80008000u) != 0) != 0, 0)) {
        add_odd(kt, buf);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) {
            v4u u = __builtin_bit_cast(v4u, v_operand(buf, ks, dt));
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint32_t e = (u[y] & 0x7C007C00u) + 0x04000400u;
              u[y] &= ~(((e >> 15) & 0x00010001u) * 0xFFFFu);
            }
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, u), pf[ks], acc[dt], 0, 0, 0);
            asm volatile("" ::: "memory");
          }
        return;
      }
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_operand(buf, ks, dt), pf[ks], acc[dt], 0, 0, 0);
    pace<16, 2, 4>();
  };

  // Phases, a barrier after each.  Of the two waves of a SIMD the second (w >= 4) is one phase
  // behind the first, so that one's products run beside the other's softmax: in step 2 j a wave
  // takes the scores of tile j and the values of tile j - 1, in step 2 j + 1 the softmax of tile j.
  // Tile j's keys are read in the phases 2 j and 2 j + 1, its values in 2 j + 2 and 2 j + 3; in
  // phase 2 i the buffers of keys i + 1 and values i are free, and the copies have until the end of
  // the next phase to land.
  // With two groups of waves (KG 2) a group's tiles are every second one, in buffers of its own.
  const auto tile_of = [&](int j) { return kt0 + KG * j + kg; };
  const auto count = [&](int end) { return max((end - kt0 - kg + KG - 1) / KG, 0); };  // of its tiles before `end`
  const int n = (kt1 - kt0 + KG - 1) / KG;                   // steps of the workgroup
  const int ng = count(kt1);                                 // tiles of the group,
  const int nw = wave_hi < 0 ? 0 : min(ng, count(wave_hi / kTile + 1));  // that a row of the wave sees a key of,
  const int nf = wave_lo < 0 ? 0 : min(nw, count((wave_lo + 1) / kTile));  // and that every row sees whole
  const auto fetch = [&](int i) __attribute__((always_inline)) {  // in phase 2 i
    if (i + 1 < ng) issue(tile_of(i + 1), (i + 1) & 1, true);
    if (i < ng) issue(tile_of(i), i & 1, false);
  };
  const auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };
  // the ends of a wave's steps 2 j and 2 j + 1
  const auto end_products = [&](int j) __attribute__((always_inline)) {
    if (late) {
      wait_vm_lgkm0<0>();
      meet();
      fetch(j + 1);
    } else {
      fetch(j);  // behind the reads: the compiler waits for copies before an LDS read
      wait_vm_lgkm0<63>();
      meet();
    }
  };
  const auto end_softmax = [&]() __attribute__((always_inline)) {
    if (!late) wait_vm_lgkm0<0>();
    meet();
  };
  if (ng > 0) issue(tile_of(0), 0, true);
  wait_vm_lgkm0<0>();
  meet();
  if (late) {
    fetch(0);
    meet();
  }
  if (nw > 0) {
    scores(0);
    end_products(0);
    softmax(tile_of(0), std::true_type{});
    end_softmax();
    int j = 1;
    const auto whole = [&](int j, int buf) __attribute__((always_inline)) {
      values(tile_of(j - 1), buf ^ 1, std::false_type{});
      scores(buf);
      end_products(j);
      softmax(tile_of(j), std::false_type{});
      end_softmax();
    };
    for (; j + 1 < nf; j += 2) {
      whole(j, 1);
      whole(j + 1, 0);
    }
    if (j < nf) {
      whole(j, 1);
      ++j;
    }
    // Tiles with keys that some row does not see.  A masked tile's values are read twice (for those
    // that are not finite), so whole ones are taken apart here too, and the one left over above:
    // 2048 tokens of 32 heads 53 -> 49 us, 16 packed prompts 447 -> 431, 37 and 4 tokens over 16000
    // and 6000 keys 39.7 -> 36.4.
    for (; j < nw; ++j) {
      if (j > nf)
        values(tile_of(j - 1), (j - 1) & 1, std::true_type{});
      else
        values(tile_of(j - 1), (j - 1) & 1, std::false_type{});
      scores(j & 1);
      end_products(j);
      softmax(tile_of(j), std::true_type{});
      end_softmax();
    }
    if (nw > nf)
      values(tile_of(nw - 1), (nw - 1) & 1, std::true_type{});
    else
      values(tile_of(nw - 1), (nw - 1) & 1, std::false_type{});
  }
  for (int j = nw; j < n; ++j) {  // other waves' tiles
    end_products(j);
    end_softmax();
  }
  if (!late) meet();

  l = halves(l, [](float x, float y) { return __fadd_rn(x, y); });
  if constexpr (KG == 2) {  // the second group's states go to the first through LDS
    float* const states = reinterpret_cast<float*>(lds);                       // [wave][64 dims][lane]
    float2* const stats = reinterpret_cast<float2*>(lds + 4 * 64 * 64 * 4);    // [wave][lane]
    uint64_t* const odds = reinterpret_cast<uint64_t*>(stats + 4 * 64);        // [wave][2][lane]
    __syncthreads();  // every wave is done with the tiles
    if (kg == 1) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) states[(rw * 64 + 16 * dt + r) * 64 + lane] = acc[dt][r];
      stats[rw * 64 + lane] = make_float2(mx, l);
      odds[rw * 128 + lane] = up;
      odds[rw * 128 + 64 + lane] = down;
    }
    __syncthreads();
    if (kg == 1) return;
    const float2 o = stats[rw * 64 + lane];
    const float M = fmaxf(mx, o.x);
    const float f0 = rescale(mx, M), f1 = rescale(o.x, M);
    mx = M;
    l = __fmaf_rn(o.y, f1, l * f0);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] = __fmaf_rn(states[(rw * 64 + 16 * dt + r) * 64 + lane], f1, acc[dt][r] * f0);
    up |= odds[rw * 128 + lane];
    down |= odds[rw * 128 + 64 + lane];
  }
  if (row >= rows) return;
  if (mx == -INFINITY && lim >= kt0 * kTile) mx = kNoScore;  // it sees a key of this part, but no score above -inf
  const float inv = SPLIT ? 1.0f : mx == -INFINITY ? 0.0f : __fdiv_rn(1.0f, l);  // a row that sees nothing is zero
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) acc[dt] *= inv;
  if (__builtin_expect(__ballot((up | down) != 0) != 0, 0)) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool u = (up >> (16 * dt + r)) & 1, d = (down >> (16 * dt + r)) & 1;
        if (u || d) acc[dt][r] += u ? (d ? NAN : INFINITY) : -INFINITY;
      }
  }
  if constexpr (SPLIT) {
    float* pr = a.part + ((qrow * a.hq + head) * a.splits + split) * kAttnPart;
    if (h == 0) {
      pr[0] = mx;
      pr[1] = l;
    }
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *reinterpret_cast<float4*>(pr + 4 + 32 * dt + 8 * y + 4 * h) =
            make_float4(acc[dt][4 * y], acc[dt][4 * y + 1], acc[dt][4 * y + 2], acc[dt][4 * y + 3]);
  } else {
    uint16_t* o = a.out + qrow * a.ldo + head * 128 + 4 * h;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *reinterpret_cast<v2u*>(o + 32 * dt + 8 * y) =
            v2u{f2h2(acc[dt][4 * y], acc[dt][4 * y + 1]), f2h2(acc[dt][4 * y + 2], acc[dt][4 * y + 3])};
  }
}

// One wave per (row of q, query head) of the sequences: the states of the parts that its tile of
// rows has, in their order.
__global__ void __launch_bounds__(64)
attn_prompt_combine(const float* part, const int32_t* cu_q, const int32_t* cu_k, uint32_t magic_hq, uint32_t magic_group, PromptArgs a) {
  const int lane = threadIdx.x;
  uint32_t t, head;
  div_rem(blockIdx.x, a.hq, magic_hq, t, head);
  int q0 = 0, n = 0, m = 0;
  bool found = false;
  for (int64_t b0 = 0; b0 < a.B && !found; b0 += 64) {
    int first = 0, rows = 0, keys = 0;
    if (b0 + lane < a.B) {  // clamped as in find_tile
      const int lq = static_cast<int>(a.Tq), lk = static_cast<int>(a.Tk);
      first = min(max(cu_q[b0 + lane], 0), lq);
      rows = max(min(cu_q[b0 + lane + 1], lq) - first, 0);
      const int k0 = min(max(cu_k[b0 + lane], 0), lk);
      keys = max(min(cu_k[b0 + lane + 1], lk) - k0, 0);
    }
    const int tt = static_cast<int>(t);
    const uint64_t in = __ballot(tt >= first && tt < first + rows);
    if (in) {
      const int f = __builtin_ctzll(in);
      q0 = __builtin_amdgcn_readlane(first, f);
      n = __builtin_amdgcn_readlane(rows, f);
      m = __builtin_amdgcn_readlane(keys, f);
      found = true;
    }
  }
  if (!found) return;  // a row of no sequence is left as it was
  // the keys of the tile of 256 rows that this row is in
  int keys = m;
  if (a.causal) {
    uint32_t hk, gh, tok, x;
    div_rem(head, a.group, magic_group, hk, gh);
    const int row = (static_cast<int>(t) - q0) * a.group + static_cast<int>(gh);
    const int last = min(row / kPromptRows * kPromptRows + kPromptRows - 1, n * a.group - 1);
    div_rem(static_cast<uint32_t>(last), a.group, magic_group, tok, x);
    keys = min(m - n + static_cast<int>(tok) + 1, m);
  }
  const int tiles = keys > 0 ? (keys + kTile - 1) / kTile : 0;
  const int per = prompt_part(tiles, a.splits, a.per);
  const int parts = max(1, (tiles + per - 1) / per);
  const float* pr = part + static_cast<int64_t>(blockIdx.x) * a.splits * kAttnPart;
  float M = -INFINITY;
  for (int s = lane; s < parts; s += 64) M = fmaxf(M, pr[static_cast<int64_t>(s) * kAttnPart]);
  M = wave_max(M);
  float L = 0.0f, D0 = 0.0f, D1 = 0.0f;
#pragma unroll 8
  for (int s = 0; s < parts; ++s) {
    const float* p = pr + static_cast<int64_t>(s) * kAttnPart;
    const float f = rescale(p[0], M);
    const float2 d = reinterpret_cast<const float2*>(p + 4)[lane];
    L = __fmaf_rn(p[1], f, L);
    D0 = __fmaf_rn(d.x, f, D0);
    D1 = __fmaf_rn(d.y, f, D1);
  }
  reinterpret_cast<uint32_t*>(a.out + t * a.ldo + static_cast<int64_t>(head) * 128)[lane] =
      M == -INFINITY ? 0u : f2h2(__fdiv_rn(D0, L), __fdiv_rn(D1, L));
}

template <bool SPLIT, int KG>
hipError_t launch_tiles(const PromptArgs& a, hipStream_t stream) {
  using P = Prompt<KG>;
  constexpr auto kern = attn_prompt_tile<SPLIT, KG>;
  const hipError_t init = set_max_lds<kern>(P::LDS);
  if (init != hipSuccess) return init;
  // as many tiles as any division of the rows among B sequences can make
  const int64_t tiles = a.Tq * a.group / P::ROWS + a.B;
  return launch(kern, dim3(static_cast<unsigned>(tiles * a.hkv * a.splits)), dim3(64 * kWaves), P::LDS, stream, a.q, a.k, a.v, a.cu_q,
                a.cu_k, div_magic(static_cast<uint32_t>(a.hkv)), div_magic(static_cast<uint32_t>(a.group)),
                div_magic(static_cast<uint32_t>(a.splits)), a);
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& a, hipStream_t stream) {
  if (a.splits == 1) return a.half ? launch_tiles<false, 2>(a, stream) : launch_tiles<false, 1>(a, stream);
  const hipError_t e = launch_tiles<true, 1>(a, stream);
  if (e != hipSuccess) return e;
  return launch(attn_prompt_combine, dim3(static_cast<unsigned>(a.Tq * a.hq)), dim3(64), 0, stream, a.part, a.cu_q, a.cu_k,
                div_magic(static_cast<uint32_t>(a.hq)), div_magic(static_cast<uint32_t>(a.group)), a);
}

}  // namespace sq
