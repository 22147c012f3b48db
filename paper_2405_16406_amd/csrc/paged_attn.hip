// Decode attention over the paged 4- or 8-bit cache with shared key/value heads: for each
// sequence b and query head h of the key/value head hk = h / group,
//     out = softmax_t(scale q . K_t) V,  K_t = ka_t c_t + kb_t (eq. 1), V_t = va_t e_t + vb_t,
//     q . K_t = ka_t (q . c_t) + kb_t sum(q),
// over the tokens t < len_b.  q . c and the weighted sum of e run on fp16 MFMA; the codes become
// fp16 without arithmetic: an integer n < 1024 in the low mantissa bits is the subnormal
// n 2^-24, which the matrix cores take as it is.  A word of eight 4-bit codes makes four pairs by
// one shift and four ands, codes 0, 2, 4, 6 as n and 1, 3, 5, 7 in place as 16 n.  The value codes
// are made normal numbers by one packed product more: see normal().
//
// A workgroup of kWaves waves serves one (sequence, key/value head, up to 16 of its query heads,
// chunk of tokens: paged_plan.h); its waves take the chunk's blocks of 64 tokens in turn, each on its own:
//   scores    S^T = K q^T by 16x16x32 products: lane (i, g) = (lane % 16, lane / 16) brings
//             bytes 16 g (4 bits) or 32 g (8 bits) .. of a token's key codes straight from
//             memory (dims 32 g .. 32 g + 31) and ends with the scores of head i for the 16
//             tokens 16 g .. 16 g + 15 of the block: products j = 0 .. 3 hold the tokens
//             16 (row / 4) + 4 j + row % 4.
//   softmax   in base 2.  V's scale goes into the weight, w_t = 2^(s_t + log2 va_t - m), with m
//             kWeightBits below the running maximum of that exponent: the fp16 weights of the second
//             product are then near 2^12 at their largest whatever the size of V.  The sums are
//             l = sum w_t / va_t and b = sum w_t vb_t / va_t in fp32.  m moves
//             (and everything is rescaled) only when the largest would grow by more than 2^kSlack.
//   values    O^T += V^T w^T: the block's value codes go through LDS as they are (64 or 128
//             bytes a token) and come back transposed (ds_read_b64_tr_b4 / _b8): lane (i, g)
//             gets the codes of dim 16 dt + i of its 16 tokens, the order its weights are in.
// HBM bounds it: a token and key/value head are 144 bytes (4 bits, fp32 parameters; 136 with fp16
// ones), or 272 with 8 bits, read once for all query heads that share them.  Each wave on its own,
// with the next block's codes in registers while one is worked on and no barrier before the end, keeps
// twelve (8 bits: eight) waves' loads in flight on a compute unit.  The arithmetic is 500 vector
// operations and 32 products a block of 4-bit codes, whether a tile has 16 heads or one: about a third
// of the time on a full device, and what is left to do when the last codes have come.  Measured, this
// kernel and the join: 131071 tokens of 8 heads, 4 bits, 31 - 33 + 4 us (151 MB: 4.6 TB/s in the
// kernel); 64 sequences of 513 .. 8192 tokens, fp16 parameters, 48 - 51 + 4 (169 MB: 3.4 TB/s); 8
// sequences of 195 .. 2048 tokens of 32 heads, 8 bits, 15 - 16 + 2; one of 2048, 8 heads, 5.5 + 1.5.
#include "paged_attn_device.h"

namespace sq {
namespace {

constexpr int kWaves = kPagedWaves;

template <int BITS>
constexpr int paged_lds() {
  const int merge = kWaves * 16 * (kDimRow + 2) * 4, codes = kWaves * WaveLds<BITS>::BYTES;
  return merge > codes ? merge : codes;
}

template <int BITS, bool P16>
__global__ void __launch_bounds__(64 * kWaves, BITS == 4 ? 3 : 2)
attn_paged_part(const uint16_t* q, const int32_t* lens, int chunks, int tiles, uint32_t magic_b, uint32_t magic_tiles,
                uint32_t magic_heads, PagedAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  using W = WaveLds<BITS>;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  // Workgroups in the order of dispatch: the chunks from a sequence's last one back are the slowest
  // index, from far to near, so that whole chunks come first and the sequences' short last ones
  // fill up at the end; then sequence, tile of heads, key/value head.
  uint32_t rest, hk, tile, b, back;
  div_rem(blockIdx.x, a.cache.heads, magic_heads, rest, hk);
  div_rem(rest, tiles, magic_tiles, rest, tile);
  div_rem(rest, static_cast<int>(a.B), magic_b, back, b);
  back = chunks - 1 - back;
  const int len = min(max(lens[b], 0), a.max_len);
  const int own = max(1, (len + a.chunk_tokens - 1) / a.chunk_tokens);  // chunks of the sequence
  if (static_cast<int>(back) >= own) return;  // the workgroup leaves together
  const int c = own - 1 - static_cast<int>(back);
  const int first = c * a.chunk_tokens;
  const int32_t* const table = a.cache.table + b * a.cache.ldt;
  const int32_t first_col = table_column(a.cache, first + w * kBlock + 16 * g);
  const int32_t first_entry = first_col < 0 ? -1 : table[first_col];
  const int last = min(len, first + a.chunk_tokens);
  const int heads = min(16, a.group - 16 * static_cast<int>(tile));  // of this workgroup
  const int h0 = static_cast<int>(hk) * a.group + 16 * static_cast<int>(tile);

  // the query of head i (rows past the heads repeat the last one and are not stored), dims
  // 32 g .. 32 g + 31, in the codes' pair order, and its sum over all dims
  v8h qf[4];
  float qsum = 0.0f;
  {
    const v4u* qv = reinterpret_cast<const v4u*>(q + b * a.ldq + static_cast<int64_t>(h0 + min(i, heads - 1)) * 128 + 32 * g);
    v4u raw[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) raw[x] = qv[x];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        qsum += h2f(static_cast<uint16_t>(raw[x][y])) + h2f(static_cast<uint16_t>(raw[x][y] >> 16));
    qsum = rows_all(qsum, [](float u, float v) { return __fadd_rn(u, v); });
    if constexpr (BITS == 4) {
      // word x holds dims 8 x ..: even products take (0, 4), (2, 6), odd ones (1, 5), (3, 7)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const v4u u = raw[2 * e], v = raw[2 * e + 1];
        qf[2 * e] = operand(__builtin_amdgcn_perm(u[2], u[0], 0x05040100u), __builtin_amdgcn_perm(u[3], u[1], 0x05040100u),
                            __builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x05040100u));
        qf[2 * e + 1] = operand(__builtin_amdgcn_perm(u[2], u[0], 0x07060302u), __builtin_amdgcn_perm(u[3], u[1], 0x07060302u),
                                __builtin_amdgcn_perm(v[2], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u));
      }
    } else {
      // a word holds dims 4 x .. 4 x + 3: pairs (0, 2) and (1, 3)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        qf[x] = operand(__builtin_amdgcn_perm(raw[x][1], raw[x][0], 0x05040100u), __builtin_amdgcn_perm(raw[x][1], raw[x][0], 0x07060302u),
                        __builtin_amdgcn_perm(raw[x][3], raw[x][2], 0x05040100u), __builtin_amdgcn_perm(raw[x][3], raw[x][2], 0x07060302u));
    }
  }

  uint8_t* const vlds = lds + w * W::BYTES;
  float* const coef = reinterpret_cast<float*>(vlds + W::CODES);
  constexpr int KW = BITS == 4 ? 1 : 2;  // 16-byte loads of a lane's key codes
  // 2^24 undoes the codes' subnormal scale
  const float cs = a.scale_log2e, cs24 = a.scale_log2e * 16777216.0f;

  v4u kc[4][KW], vc[4][KW];
  float4 par;
  bool par_ok;
  // A block's pages: each lane holds that of its 16-token group, lane / 16 (pages hold 16 tokens or
  // more, so a group lies in one).  The table entry is read a block ahead of the codes, and for the
  // first block beside the length.
  auto entry_of = [&](int t0) -> int32_t {
    const int32_t col = table_column(a.cache, t0 + 16 * g);
    return col < 0 ? -1 : table[col];
  };
  auto load = [&](int t0, int32_t entry) __attribute__((always_inline)) {
    // tokens without a page, or past the chunk, read page 0 and are masked below
    const int32_t mine = valid_page(a.cache, entry);
    par_ok = mine >= 0 && t0 + lane < last;
    const int32_t safe = max(mine, 0);
    int32_t pg[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) pg[n] = __builtin_amdgcn_readlane(safe, 16 * n);
    const int n = i >> 2;  // keys: the lane's token is one of group i / 4
    const int32_t pk = n == 0 ? pg[0] : n == 1 ? pg[1] : n == 2 ? pg[2] : pg[3];
    const uint8_t* kp = a.cache.kq + token_slot(a.cache, pk, hk, t0 + 16 * n + (i & 3)) * W::ROW + (BITS == 4 ? 16 : 32) * g;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int x = 0; x < KW; ++x) kc[j][x] = *reinterpret_cast<const v4u*>(kp + 4 * j * W::ROW + 16 * x);
    // values: load m brings group m, four (eight) lanes a token
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const uint8_t* vp = a.cache.vq + token_slot(a.cache, pg[m], hk, t0 + 16 * m) * W::ROW + 16 * lane;
#pragma unroll
      for (int x = 0; x < KW; ++x) vc[m][x] = *reinterpret_cast<const v4u*>(vp + 1024 * x);
    }
    // parameters: lane's token is t0 + lane
    const int64_t pslot = token_slot(a.cache, safe, hk, t0 + lane);
    if constexpr (P16) {
      const uint2 p = static_cast<const uint2*>(a.cache.params)[pslot];
      par = make_float4(h2f(static_cast<uint16_t>(p.x)), h2f(static_cast<uint16_t>(p.x >> 16)),
                        h2f(static_cast<uint16_t>(p.y)), h2f(static_cast<uint16_t>(p.y >> 16)));
    } else {
      par = static_cast<const float4*>(a.cache.params)[pslot];
    }
  };

  float m = -INFINITY, l = 0.0f, bsum = 0.0f;
  uint64_t seen = 0;  // lanes that had a token with a page
  v4f acc[8];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  const int step = kWaves * kBlock;
  int t0 = first + w * kBlock;
  int32_t entry = -1;
  if (t0 < last) {
    load(t0, first_entry);
    entry = entry_of(t0 + step);
  }
  for (; t0 < last; t0 += step) {
    // value codes and coefficients to LDS (this wave's own: no barrier, its LDS operations are
    // in order); unit u of a row of 4 (8) units lies at u xor (row / 4) % 4 (u xor row % 8)
#pragma unroll
    for (int mm = 0; mm < 4; ++mm)
#pragma unroll
      for (int x = 0; x < KW; ++x) {
        const int row = 16 * mm + (BITS == 4 ? lane >> 2 : 8 * x + (lane >> 3));  // 16 bytes a lane, in order
        const int unit = BITS == 4 ? (lane & 3) ^ ((row >> 2) & 3) : (lane & 7) ^ (row & 7);
        *reinterpret_cast<v4u*>(vlds + row * W::ROW + 16 * unit) = vc[mm][x];
      }
    seen |= __ballot(par_ok);
    // A slot of a zeroed cache that was never written: its codes are 0, so any scale gives its values.
    // (Codes of such tokens are not looked at: a branch that clears them in LDS costs 3 % and a spill.)
    par.z = par.z == 0.0f ? 1.0f : par.z;
    const float rva = par_ok ? __fdiv_rn(1.0f, par.z) : 0.0f;
    coef[0 * kBlock + lane] = par_ok ? par.x * cs24 : 0.0f;
    coef[1 * kBlock + lane] = par_ok ? par.y * cs : 0.0f;
    coef[2 * kBlock + lane] = par_ok ? __builtin_amdgcn_logf(par.z) : -INFINITY;
    coef[3 * kBlock + lane] = rva;
    coef[4 * kBlock + lane] = par_ok ? par.w * rva : 0.0f;
    v4u kn[4][KW];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int x = 0; x < KW; ++x) kn[j][x] = kc[j][x];
    if (t0 + step < last) {
      load(t0 + step, entry);
      entry = entry_of(t0 + 2 * step);
    }
    asm volatile("" ::: "memory");

    // scores of 16 tokens of head i
    float s[16];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 ca = *reinterpret_cast<const float4*>(coef + 0 * kBlock + 16 * g + 4 * j);
      const float4 cb = *reinterpret_cast<const float4*>(coef + 1 * kBlock + 16 * g + 4 * j);
      const float4 cl = *reinterpret_cast<const float4*>(coef + 2 * kBlock + 16 * g + 4 * j);
      const float* fa = &ca.x;
      const float* fb = &cb.x;
      const float* fl = &cl.x;
      v4f se = {0.0f, 0.0f, 0.0f, 0.0f}, so = {0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (BITS == 4) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t u = kn[j][0][2 * e], v = kn[j][0][2 * e + 1], u8 = u >> 8, v8 = v >> 8;
          se = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              operand(u & 0x000F000Fu, u8 & 0x000F000Fu, v & 0x000F000Fu, v8 & 0x000F000Fu), qf[2 * e], se, 0, 0, 0);
          so = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              operand(u & 0x00F000F0u, u8 & 0x00F000F0u, v & 0x00F000F0u, v8 & 0x00F000F0u), qf[2 * e + 1], so, 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t u = kn[j][x / 2][2 * (x & 1)], v = kn[j][x / 2][2 * (x & 1) + 1];
          v4f& acc_s = x & 1 ? so : se;
          acc_s = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              operand(u & 0x00FF00FFu, (u >> 8) & 0x00FF00FFu, v & 0x00FF00FFu, (v >> 8) & 0x00FF00FFu), qf[x], acc_s, 0, 0, 0);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float dot = BITS == 4 ? __fmaf_rn(so[r], 0.0625f, se[r]) : __fadd_rn(se[r], so[r]);
        s[4 * j + r] = __fmaf_rn(fa[r], dot, __fmaf_rn(fb[r], qsum, fl[r]));
        top = fmaxf(top, s[4 * j + r]);
      }
    }
    top = rows_all(top, [](float u, float v) { return fmaxf(u, v); });
    if (__ballot(top - m > kWeightBits + kSlack)) {  // (m = -inf: any token)
      const float mn = fmaxf(m, fabsf(top) < kLargeScore ? top - kWeightBits : top);
      const float f = rescale(m, mn);
      l *= f;
      bsum *= f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[dt] *= f;
      m = mn;
    }
    // Weights in the value codes' pair order, rounded to fp16.  l and b sum the rounded ones: their
    // rounding then moves the mean of the values seen by 2^-12 of their spread; against unrounded
    // sums it would be 2^-12 of sum w e, whose bulk cancels against b (errors of the output 0.4 -
    // 0.8e-3 over long caches instead of 0.2 - 0.3e-3).
    const float base = m == -INFINITY ? 0.0f : m;
    uint32_t pw[8];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float4 cr0 = *reinterpret_cast<const float4*>(coef + 3 * kBlock + 16 * g + 8 * x);
      const float4 cr1 = *reinterpret_cast<const float4*>(coef + 3 * kBlock + 16 * g + 8 * x + 4);
      const float4 cv0 = *reinterpret_cast<const float4*>(coef + 4 * kBlock + 16 * g + 8 * x);
      const float4 cv1 = *reinterpret_cast<const float4*>(coef + 4 * kBlock + 16 * g + 8 * x + 4);
      const float fr[8] = {cr0.x, cr0.y, cr0.z, cr0.w, cr1.x, cr1.y, cr1.z, cr1.w};
      const float fv[8] = {cv0.x, cv0.y, cv0.z, cv0.w, cv1.x, cv1.y, cv1.z, cv1.w};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        // pairs of tokens: 4 bits (0, 4), (1, 5), (2, 6), (3, 7); 8 bits (0, 2), (1, 3), ..
        const int t0 = BITS == 4 ? y : 4 * (y >> 1) + (y & 1), t1 = t0 + (BITS == 4 ? 4 : 2);
        const uint32_t p2 = f2h2(exp2_fast(s[8 * x + t0] - base), exp2_fast(s[8 * x + t1] - base));
        pw[4 * x + y] = p2;
        const v2h ph = __builtin_bit_cast(v2h, p2);
        l = __fmaf_rn(static_cast<float>(ph[0]), fr[t0], l);
        l = __fmaf_rn(static_cast<float>(ph[1]), fr[t1], l);
        bsum = __fmaf_rn(static_cast<float>(ph[0]), fv[t0], bsum);
        bsum = __fmaf_rn(static_cast<float>(ph[1]), fv[t1], bsum);
      }
    }
    const v8h pf[2] = {operand(pw[0], pw[1], pw[2], pw[3]), operand(pw[4], pw[5], pw[6], pw[7])};
    typedef __attribute__((address_space(3))) v2i* lds_v2i;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      if constexpr (BITS == 4) {
        const int row = 16 * g + i;
        const uint8_t* p = vlds + row * W::ROW + 16 * ((dt >> 1) ^ ((row >> 2) & 3)) + 8 * (dt & 1);
        const v2i c2 = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_v2i)(uintptr_t)(p));
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t u = static_cast<uint32_t>(c2[x]), u8 = u >> 8;
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(normal(u & 0x000F000Fu, 0), normal(u & 0x00F000F0u, 4),
                                                                   normal(u8 & 0x000F000Fu, 0), normal(u8 & 0x00F000F0u, 4)),
                                                           pf[x], acc[dt], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = 16 * g + 8 * x + (i >> 1);
          const uint8_t* p = vlds + row * W::ROW + 16 * (dt ^ (row & 7)) + 8 * (i & 1);
          const v2i c2 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i)(uintptr_t)(p));
          const uint32_t u = static_cast<uint32_t>(c2[0]), v = static_cast<uint32_t>(c2[1]);
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              operand(normal(u & 0x00FF00FFu, 0), normal((u >> 8) & 0x00FF00FFu, 0),
                      normal(v & 0x00FF00FFu, 0), normal((v >> 8) & 0x00FF00FFu, 0)),
              pf[x], acc[dt], 0, 0, 0);
        }
      }
    }
    asm volatile("" ::: "memory");
  }
  const auto add = [](float u, float v) { return __fadd_rn(u, v); };
  l = rows_all(l, add);
  bsum = rows_all(bsum, add);
  if (seen == 0) {  // masked tokens alone: a query that is not finite has made their sums NaN
    m = -INFINITY;
    l = bsum = 0.0f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  } else if (m == -INFINITY) {
    m = kNoScore;
  }

  // the waves' states of each head meet in LDS: dims finished but for the division
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);                  // [wave][head][kDimRow]
  float* const red_ml = red + kWaves * 16 * kDimRow;                 // [wave][head][2]
  if (g == 0) {
    red_ml[(w * 16 + i) * 2] = m;
    red_ml[(w * 16 + i) * 2 + 1] = l;
  }
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    v4f o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = __fmaf_rn(acc[dt][r], 512.0f, bsum);
    *reinterpret_cast<v4f*>(red + (w * 16 + i) * kDimRow + 16 * dt + 4 * g) = o;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < heads * 32; x += 64 * kWaves) {
    const int hh = x >> 5, d = 4 * (x & 31);
    float M = -INFINITY;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) M = fmaxf(M, red_ml[(v * 16 + hh) * 2]);
    float L = 0.0f;
    v4f D = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float f = rescale(red_ml[(v * 16 + hh) * 2], M);
      L = __fmaf_rn(red_ml[(v * 16 + hh) * 2 + 1], f, L);
      const v4f o = *reinterpret_cast<const v4f*>(red + (v * 16 + hh) * kDimRow + d);
#pragma unroll
      for (int r = 0; r < 4; ++r) D[r] = __fmaf_rn(o[r], f, D[r]);
    }
    const int64_t head = h0 + hh;
    if (own == 1) {
      uint16_t* o = a.out + b * a.ldo + head * 128 + d;
      if (M == -INFINITY)  // no token
        *reinterpret_cast<v2u*>(o) = v2u{0u, 0u};
      else
        *reinterpret_cast<v2u*>(o) = v2u{f2h2(__fdiv_rn(D[0], L), __fdiv_rn(D[1], L)), f2h2(__fdiv_rn(D[2], L), __fdiv_rn(D[3], L))};
    } else {
      float* pr = a.part + ((b * static_cast<int64_t>(a.hq) + head) * chunks + c) * kAttnPart;
      if (d == 0) {
        pr[0] = M;
        pr[1] = L;
      }
      *reinterpret_cast<v4f*>(pr + 4 + d) = D;
    }
  }
}

// One workgroup per (sequence, query head) with more than one chunk: wave w adds the chunks w, w + J,
// ..., then the waves' sums are added in their order.
template <int J>
__global__ void __launch_bounds__(64 * J)
attn_paged_combine(const float* part, const int32_t* lens, uint16_t* out, int64_t ldo, int hq, int chunks, int chunk_tokens,
                   int max_len, uint32_t magic_hq) {
  __shared__ float red_m[J], red_l[J];
  __shared__ float2 red_d[J][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t b, h;
  div_rem(blockIdx.x, hq, magic_hq, b, h);
  const int len = min(max(lens[b], 0), max_len);
  const int n = (len + chunk_tokens - 1) / chunk_tokens;
  if (n <= 1) return;  // its workgroup has written the output
  const float* pr = part + (b * static_cast<int64_t>(hq) + h) * chunks * kAttnPart;
  float M = -INFINITY, L = 0.0f, D0 = 0.0f, D1 = 0.0f;
  constexpr int kAhead = 8;  // chunks whose loads are in flight together
  for (int c0 = w; c0 < n; c0 += J * kAhead) {
    float2 ml[kAhead], d[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {  // a chunk past the last is the last again, with weight 0
      const float* p = pr + static_cast<int64_t>(min(c0 + J * x, n - 1)) * kAttnPart;
      ml[x] = *reinterpret_cast<const float2*>(p);
      d[x] = reinterpret_cast<const float2*>(p + 4)[lane];
    }
    float top = M;
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      if (c0 + J * x >= n) ml[x].x = -INFINITY;
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
  reinterpret_cast<uint32_t*>(out + b * ldo + static_cast<int64_t>(h) * 128)[lane] =
      M == -INFINITY ? 0u : f2h2(__fdiv_rn(D0, L), __fdiv_rn(D1, L));
}

template <int BITS, bool P16>
hipError_t launch_part(const PagedAttnArgs& a, hipStream_t stream) {
  constexpr auto kern = attn_paged_part<BITS, P16>;
  constexpr int lds = paged_lds<BITS>();
  const hipError_t init = set_max_lds<kern>(lds);
  if (init != hipSuccess) return init;
  const int tiles = (a.group + 15) / 16;
  const unsigned blocks = static_cast<unsigned>(a.B * a.cache.heads * tiles * a.chunks);
  return launch(kern, dim3(blocks), dim3(64 * kWaves), lds, stream, a.q, a.lens, a.chunks, tiles,
                div_magic(static_cast<uint32_t>(a.B)), div_magic(static_cast<uint32_t>(tiles)),
                div_magic(static_cast<uint32_t>(a.cache.heads)), a);
}

}  // namespace

hipError_t launch_attn_paged(const PagedAttnArgs& a, hipStream_t stream) {
  hipError_t e;
  if (a.bits == 8)
    e = a.param16 ? launch_part<8, true>(a, stream) : launch_part<8, false>(a, stream);
  else
    e = a.param16 ? launch_part<4, true>(a, stream) : launch_part<4, false>(a, stream);
  if (e != hipSuccess || a.chunks == 1) return e;
  const auto join = [&](auto kern, int waves) {
    return launch(kern, dim3(static_cast<unsigned>(a.B * a.hq)), dim3(64 * waves), 0, stream, a.part, a.lens, a.out, a.ldo, a.hq,
                  a.chunks, a.chunk_tokens, a.max_len, div_magic(static_cast<uint32_t>(a.hq)));
  };
  // (4096 heads of 64 sequences in two chunks: 4 us less with one wave each than with eight)
  return a.chunks <= 8 ? join(attn_paged_combine<1>, 1) : join(attn_paged_combine<8>, 8);
}

}  // namespace sq
