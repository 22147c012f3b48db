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
//   softmax  in base 2, running maximum m and sum l in fp32.  m moves, and the output is rescaled,
//            only where it would grow by more than kSlack.
//   values   O^T += V^T P^T.  The slots of the product's inner index may hold the keys in any
//            order, the same for both operands: in the order in which the first product leaves
//            the scores, the rounded weights are an operand as they are; V comes from LDS by
//            transposed reads (ds_read_b64_tr_b16) of the same keys.
// Tiles of K and V go from memory straight to LDS, one ahead of the products.  A tile's row is 256
// bytes; its 16-byte chunk c lies at c xor swizzle(row), so that neither the 16 rows of a K read
// nor the 4 x 64 bytes of a transposed read of V meet on a bank.
// Weights are rounded to fp16 (2^-12 of the weight, as the output is); sums stay in fp32.
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
constexpr int kLds = 4 * kTileBytes;        // two tiles of each
constexpr float kSlack = 8.0f;              // log2: weights stay below 2^(kWeightBits + kSlack) < 65504
constexpr float kWeightBits = 7.0f;         // the largest weight when m has just moved
static_assert(kPromptRows == 32 * kWaves, "a wave owns 32 rows");

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

// Sequence and tile of the tile number `rem` among ceil(rows / 256) tiles a sequence.
struct PromptTile {
  int seq;          // -1: past the last
  int tile, tiles;
  int q0, n;        // first row of q and rows of the sequence
};
__device__ __forceinline__ PromptTile find_tile(const int32_t* cu_q, int64_t B, int64_t Tq, int group, int rem) {
  const int lane = threadIdx.x & 63;
  for (int64_t b0 = 0; b0 < B; b0 += 64) {
    int q0 = 0, n = 0;
    if (b0 + lane < B) {  // clamped to the tensor, whatever cu_q holds
      const int last = static_cast<int>(Tq);
      q0 = min(max(cu_q[b0 + lane], 0), last);
      n = max(min(cu_q[b0 + lane + 1], last) - q0, 0);
    }
    const int tiles = (n * group + kPromptRows - 1) / kPromptRows;
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    const uint64_t past = __ballot(upto > rem);
    if (past) {
      const int f = __builtin_ctzll(past);
      const int t = __builtin_amdgcn_readlane(tiles, f);
      return {static_cast<int>(b0) + f, rem - (__builtin_amdgcn_readlane(upto, f) - t), t, __builtin_amdgcn_readlane(q0, f),
              __builtin_amdgcn_readlane(n, f)};
    }
    rem -= __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0, 0, 0, 0};
}

template <bool SPLIT>
__global__ void __launch_bounds__(64 * kWaves, 2)
attn_prompt_tile(const uint16_t* q, const uint16_t* k, const uint16_t* v, const int32_t* cu_q, const int32_t* cu_k,
                 uint32_t magic_heads, uint32_t magic_group, uint32_t magic_splits, PromptArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  uint32_t rest, hk, split = 0;
  div_rem(blockIdx.x, a.hkv, magic_heads, rest, hk);
  if constexpr (SPLIT) {
    uint32_t r2;
    div_rem(rest, a.splits, magic_splits, r2, split);
    rest = r2;
  }
  const PromptTile pt = find_tile(cu_q, a.B, a.Tq, a.group, static_cast<int>(rest));
  if (pt.seq < 0) return;  // the workgroup leaves together
  const int tile = a.causal ? pt.tiles - 1 - pt.tile : pt.tile;  // the longest first
  const int k0 = min(max(cu_k[pt.seq], 0), static_cast<int>(a.Tk));
  const int m = max(min(cu_k[pt.seq + 1], static_cast<int>(a.Tk)) - k0, 0);
  const int rows = pt.n * a.group;

  // this lane's row: rows past the last repeat it and are not stored
  const int row = tile * kPromptRows + 32 * w + col;
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
  const int wave_lo = limit(tile * kPromptRows + 32 * w), wave_hi = limit(tile * kPromptRows + 32 * w + 31);
  const int keys = limit(tile * kPromptRows + kPromptRows - 1) + 1;  // of the workgroup
  const int tiles_all = keys > 0 ? (keys + kTile - 1) / kTile : 0;
  int kt0 = 0, kt1 = tiles_all;
  if constexpr (SPLIT) {
    const int per = (tiles_all + a.splits - 1) / a.splits;
    kt0 = min(static_cast<int>(split) * per, tiles_all);
    kt1 = min(kt0 + per, tiles_all);
  }

  // Q^T operands: lane (row, h) holds dims 16 s + 8 h .. + 7
  v8h qf[8];
  {
    const uint16_t* qp = q + qrow * a.ldq + head * 128 + 8 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const v8h*>(qp + 16 * s);
  }

  // copies: instruction x of a tile brings rows 4 x .. 4 x + 3; wave w takes x = 2 w, 2 w + 1 of K
  // and of V
  const int ldk2 = static_cast<int>(a.ldk * 2), ldv2 = static_cast<int>(a.ldv * 2);
  int koff[2], voff[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int r = 4 * (2 * w + x) + (lane >> 4);
    const int c = (lane & 15) ^ swizzle(r);
    koff[x] = r * ldk2 + 16 * c;
    voff[x] = r * ldv2 + 16 * c;
  }
  const uint8_t* const kbase = reinterpret_cast<const uint8_t*>(k + k0 * a.ldk + static_cast<int64_t>(hk) * 128);
  const uint8_t* const vbase = reinterpret_cast<const uint8_t*>(v + k0 * a.ldv + static_cast<int64_t>(hk) * 128);
  typedef __attribute__((address_space(3))) void* lds_ptr;
  auto issue = [&](int kt, int buf) {
    // rows past the last key are out of the buffer and land as zeros
    const int n = min(kTile, m - kt * kTile);
    const __amdgpu_buffer_rsrc_t rk = buf_rsrc(kbase + static_cast<int64_t>(kt) * kTile * ldk2, static_cast<int64_t>(n - 1) * ldk2 + 256);
    const __amdgpu_buffer_rsrc_t rv = buf_rsrc(vbase + static_cast<int64_t>(kt) * kTile * ldv2, static_cast<int64_t>(n - 1) * ldv2 + 256);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint8_t* dst = lds + buf * kTileBytes + (2 * w + x) * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_ptr)(uintptr_t)dst, 16, koff[x], 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_ptr)(uintptr_t)(dst + 2 * kTileBytes), 16, voff[x], 0, 0, 0);
    }
  };

  // LDS reads: K row `col` of each half tile, chunk 2 s + h; V: lane (i, gi) of 16 reads 8 bytes of
  // row 4 h + i / 4 (+ 8), dims 32 dt + 16 (gi % 2) + 4 (i % 4) .. and gets dim 32 dt + col of four keys
  const int ksw = swizzle(col);
  const int vrow = 4 * h + ((lane & 15) >> 2), vlow = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), vsub = 8 * (lane & 1);
  auto v_read = [&](int buf, int ks, int dt, int second) -> v4s {
    const int t = vrow + 8 * second;
    const int off = (2 + buf) * kTileBytes + ks * 16 * 256 + t * 256 + 16 * ((4 * dt + vlow) ^ swizzle(t)) + vsub;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)(lds + off));
  };
  auto v_operand = [&](int buf, int ks, int dt) -> v8h {
    const v4s x = v_read(buf, ks, dt, 0), y = v_read(buf, ks, dt, 1);
    return __builtin_bit_cast(v8h, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  float mx = -INFINITY, l = 0.0f;
  v16f acc[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[dt][r] = 0.0f;
  const float cs = a.scale_log2e;

  auto step = [&](int kt, int buf) {
    v16f s[2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = 0.0f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const v8h kf = *reinterpret_cast<const v8h*>(lds + buf * kTileBytes + (32 * mt + col) * 256 + 16 * ((2 * x + h) ^ ksw));
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[x], s[mt], 0, 0, 0);
      }
    }
    // keys 64 kt + 32 mt + 8 (r / 4) + 4 h + r % 4
    const bool masked = kt * kTile + kTile - 1 > wave_lo;  // uniform over the wave
    if (masked) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (kt * kTile + 32 * mt + 8 * (r >> 2) + 4 * h + (r & 3) > lim) s[mt][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[0][r]);
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[1][r]);
    top = halves(top, [](float x, float y) { return fmaxf(x, y); }) * cs;
    if (__ballot(top > mx + kSlack)) {  // (mx = -inf: any score)
      const float mn = fmaxf(mx, top);
      const float f = rescale(mx, mn);
      l *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) acc[dt] *= f;
      mx = mn;
    }
    const float base = (mx == -INFINITY ? 0.0f : mx) - kWeightBits;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[mt][r] = exp2_fast(__fmaf_rn(s[mt][r], cs, -base));
        l += s[mt][r];
      }
    v8h pf[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      uint32_t p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = f2h2(s[ks >> 1][8 * (ks & 1) + 2 * r], s[ks >> 1][8 * (ks & 1) + 2 * r + 1]);
      pf[ks] = __builtin_bit_cast(v8h, v4u{p[0], p[1], p[2], p[3]});
    }
    // A weight of 0 does not hide a value that is not finite, and in a masked tile some rows must
    // not see what others do: there, such values are taken out of the product and added by hand.
    if (masked) {
      uint32_t odd = 0;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          const v4u u = __builtin_bit_cast(v4u, v_operand(buf, ks, dt));
#pragma unroll
          for (int y = 0; y < 4; ++y) odd |= (u[y] & 0x7C007C00u) + 0x04000400u;
        }
      if (__ballot((odd & 0x80008000u) != 0)) {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) {
            v4u u = __builtin_bit_cast(v4u, v_operand(buf, ks, dt));
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint32_t e = (u[y] & 0x7C007C00u) + 0x04000400u;
              if (e & 0x8000u) u[y] &= 0xFFFF0000u;
              if (e & 0x80000000u) u[y] &= 0x0000FFFFu;
            }
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, u), pf[ks], acc[dt], 0, 0, 0);
          }
        for (int t = 0; t < kTile; ++t) {
          if (kt * kTile + t > lim) continue;
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const v2u u = *reinterpret_cast<const v2u*>(lds + (2 + buf) * kTileBytes + t * 256 + 16 * ((4 * dt + y) ^ swizzle(t)) + 8 * h);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint16_t x = static_cast<uint16_t>(u[e >> 1] >> (16 * (e & 1)));
                if ((x & 0x7C00u) == 0x7C00u) acc[dt][4 * y + e] += h2f(x);
              }
            }
        }
        return;
      }
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_operand(buf, ks, dt), pf[ks], acc[dt], 0, 0, 0);
  };

  if (kt0 < kt1) issue(kt0, 0);
  for (int kt = kt0; kt < kt1; kt += 2) {
    static_for<2>([&](auto bc) {
      constexpr int buf = decltype(bc)::value;
      if (kt + buf < kt1) {  // uniform over the workgroup
        wait_vm_lgkm0<0>();  // this wave's part of tile kt + buf has landed
        __syncthreads();     // every part has; and every wave is done with the other buffer
        if (kt + buf + 1 < kt1) issue(kt + buf + 1, buf ^ 1);
        if ((kt + buf) * kTile <= wave_hi) step(kt + buf, buf);
      }
    });
  }

  l = halves(l, [](float x, float y) { return __fadd_rn(x, y); });
  if (row >= rows) return;
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
    const float inv = mx == -INFINITY ? 0.0f : __fdiv_rn(1.0f, l);  // a row that sees nothing is zero
    uint16_t* o = a.out + qrow * a.ldo + head * 128 + 4 * h;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *reinterpret_cast<v2u*>(o + 32 * dt + 8 * y) =
            v2u{f2h2(acc[dt][4 * y] * inv, acc[dt][4 * y + 1] * inv), f2h2(acc[dt][4 * y + 2] * inv, acc[dt][4 * y + 3] * inv)};
  }
}

// One wave per (row of q, query head) of the sequences: the splits' states, in their order.
__global__ void __launch_bounds__(64)
attn_prompt_combine(const float* part, const int32_t* cu_q, int64_t B, int hq, int splits, uint32_t magic_hq, uint16_t* out,
                    int64_t ldo) {
  const int lane = threadIdx.x;
  uint32_t t, head;
  div_rem(blockIdx.x, hq, magic_hq, t, head);
  if (find_sequence(cu_q, B, t).seq < 0) return;  // a row of no sequence is left as it was
  const float* pr = part + static_cast<int64_t>(blockIdx.x) * splits * kAttnPart;
  float M = -INFINITY;
  for (int s = lane; s < splits; s += 64) M = fmaxf(M, pr[static_cast<int64_t>(s) * kAttnPart]);
  M = wave_max(M);
  float L = 0.0f, D0 = 0.0f, D1 = 0.0f;
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float* p = pr + static_cast<int64_t>(s) * kAttnPart;
    const float f = rescale(p[0], M);
    const float2 d = reinterpret_cast<const float2*>(p + 4)[lane];
    L = __fmaf_rn(p[1], f, L);
    D0 = __fmaf_rn(d.x, f, D0);
    D1 = __fmaf_rn(d.y, f, D1);
  }
  reinterpret_cast<uint32_t*>(out + t * ldo + static_cast<int64_t>(head) * 128)[lane] =
      M == -INFINITY ? 0u : f2h2(__fdiv_rn(D0, L), __fdiv_rn(D1, L));
}

template <bool SPLIT>
hipError_t launch_tiles(const PromptArgs& a, hipStream_t stream) {
  constexpr auto kern = attn_prompt_tile<SPLIT>;
  const hipError_t init = set_max_lds<kern>(kLds);
  if (init != hipSuccess) return init;
  // as many tiles as any division of the rows among B sequences can make
  const int64_t tiles = a.Tq * a.group / kPromptRows + a.B;
  return launch(kern, dim3(static_cast<unsigned>(tiles * a.hkv * a.splits)), dim3(64 * kWaves), kLds, stream, a.q, a.k, a.v, a.cu_q,
                a.cu_k, div_magic(static_cast<uint32_t>(a.hkv)), div_magic(static_cast<uint32_t>(a.group)),
                div_magic(static_cast<uint32_t>(a.splits)), a);
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& a, hipStream_t stream) {
  if (a.splits == 1) return launch_tiles<false>(a, stream);
  const hipError_t e = launch_tiles<true>(a, stream);
  if (e != hipSuccess) return e;
  return launch(attn_prompt_combine, dim3(static_cast<unsigned>(a.Tq * a.hq)), dim3(64), 0, stream, a.part, a.cu_q, a.B, a.hq,
                a.splits, div_magic(static_cast<uint32_t>(a.hq)), a.out, a.ldo);
}

}  // namespace sq
