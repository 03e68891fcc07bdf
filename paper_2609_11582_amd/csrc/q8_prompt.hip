// Attention of many rows over the paged 8-bit cache: chunks and whole prompts.
//
// The formulas are the split kernel's (q8_attention.hip); here the products dominate: 4 x 128 flops a row and token,
// far above what the 256 bytes of a token cost. A work-group takes 256 query columns (the G heads of consecutive
// positions), 8 waves of 32, and walks the tokens in tiles of 64:
//  * Codes are widened to fp16 once a tile and work-group, on their way from memory through registers to LDS (two
//    buffers: the next tile is written while one is used, the one after is in flight). Both kinds lie in LDS as
//    the 32x32x16 matrix instructions' A operands, 1 KB each, so every read is 64 lanes x 16 contiguous bytes.
//  * Scores: rows = 32 tokens, columns = queries, the query held in registers. A lane holds half the tokens of one
//    column, so the softmax is in-lane but for one exchange of maxima; the weights are the value product's B operand
//    as they stand (k slot of step s, half h, 4 a + i <-> token 16 a + 8 s + 4 h + i, which is also the order of 8
//    consecutive bytes of a value block).
//  * The weights are formed in one fused step as 2^(dot * scale + c), c = log2 v_scale + 7 - M; their sum, divided
//    by the block's factor, is the block's share of the softmax sum.
// Bound: the exponentials and the matrix instructions, in turn (about 900 cycles of VALU work to 1024 of matrix work
// a wave and tile).
#include <algorithm>

#include "q8_mfma.hpp"

namespace okvq {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 64;                 // tokens
constexpr int kOperand = 64;              // 16-byte slots of a matrix operand
static_assert(kQ8PromptCols == 32 * kWaves, "32 columns a wave");

struct Tile {                             // one buffer
  uint4 k[2][8][kOperand];                // [block][16 channels][half h, token]: token's place is token ^ (channels & 7)
  uint4 v[2][4][2][kOperand];             // [block][32 channels][step s][half h, channel]
  float ks[2], vs[2];
};
struct Raw {                              // a thread's 16 bytes of keys and of values
  uint4 k, v;
  float ks, vs;
};

template <int kFmt, bool kBf16>
__global__ __launch_bounds__(kThreads) void k_q8_prompt(Q8AttendArgs p, int B) {
  __shared__ Tile buf[2];
  const Q8View& c = p.c;
  // sequences and heads vary fastest: work-groups go round the 8 XCDs, so a head's tiles meet in few L2s; the last rows,
  // which see most, start first
  const int units = B * c.H, unit = blockIdx.x % units, split = blockIdx.y;
  const int tile = p.ntile - 1 - (int)(blockIdx.x / units), b = unit / c.H, h = unit - b * c.H;
  const int first = p.splits.first[b], records = p.splits.first[b + 1] - first, nsplit = max(records, 1);
  if (split >= nsplit) return;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* table = c.table + (int64_t)b * c.max_pages;
  const int len = q8_len(c, b), n = min(max(uniform_load(p.n_new + b), 0), p.n_max);
  const int r0 = tile * kQ8PromptCols, i_first = r0 / p.G;
  if (i_first >= n) return;
  const int i_last = min((r0 + kQ8PromptCols - 1) / p.G, n - 1);
  const int vis_last = p.cross ? len : max(len - n + i_last + 1, 0);
  // the wave's columns, and the tokens that they see
  const int r = r0 + 32 * wave + col, i = r / p.G, hq = h * p.G + (r - i * p.G);
  const bool live = i < n;
  const int vis = live ? (p.cross ? len : max(len - n + i + 1, 0)) : 0;
  const int wave_first = (r0 + 32 * wave) / p.G;
  const int vis_first = wave_first >= n ? 0 : p.cross ? len : max(len - n + wave_first + 1, 0);
  const int ntile = (vis_last + kTile - 1) / kTile;
  const int per = (ntile + nsplit - 1) / nsplit, t_begin = min(split * per, ntile), t_end = min(t_begin + per, ntile);

  // staging: thread tid has 16 bytes of key row tid / 8 and value slot tid % 256 of block tid / 256
  const int sb = wave >> 2, krow = (tid >> 3) & 31, kchunk = tid & 7, vslot = tid & 255;
  int page = q8_page(table, 2 * t_begin + sb, c);
  auto load = [&](int t, Raw& x) {
    const int block = 2 * t + sb;  // may lie behind the sequence: then codes of any page inside the pool, all masked
    const int64_t slot = q8_slot(page, h, block, c);
    x.k = *reinterpret_cast<const uint4*>(c.k_codes + slot * kQ8Block + vslot * 16);
    x.v = *reinterpret_cast<const uint4*>(c.v_codes + slot * kQ8Block + vslot * 16);
    x.ks = uniform_load(c.k_scale + slot);
    x.vs = uniform_load(c.v_scale + slot);
    page = q8_page(table, block + 2, c);  // of the next call's block
    if (block * kW >= len) {  // what is multiplied by a zero weight has to be finite
      x.k = x.v = make_uint4(0u, 0u, 0u, 0u);
      x.ks = x.vs = 1.0f;
    }
  };
  auto store = [&](Tile& t, const Raw& x) {
    const int kp = krow ^ kchunk;
    t.k[sb][kchunk][kp] = __builtin_bit_cast(uint4, widen8<kFmt>(x.k.x, x.k.y));
    t.k[sb][kchunk][32 + kp] = __builtin_bit_cast(uint4, widen8<kFmt>(x.k.z, x.k.w));
    const int j = vslot >> 6, g = (vslot >> 4) & 3, ch = vslot & 15;
    t.v[sb][j][g >> 1][32 * (g & 1) + ch] = __builtin_bit_cast(uint4, widen8<kFmt>(x.v.x, x.v.y));
    t.v[sb][j][g >> 1][32 * (g & 1) + 16 + ch] = __builtin_bit_cast(uint4, widen8<kFmt>(x.v.z, x.v.w));
    if (krow == 0 && kchunk == 0) {
      t.ks[sb] = x.ks;
      t.vs[sb] = x.vs;
    }
  };

  // query operands: column's channels 16 kk + 8 half .. + 7
  half8 qop[8];
  float qs = fabsf(p.qscale);
  {
    const uint4* q = reinterpret_cast<const uint4*>(p.q) + (((int64_t)b * c.Hq + hq) * p.n_max + i) * 16 + half;
    uint4 raw[8];
    const uint32_t flip = p.qscale < 0.0f ? 0x80008000u : 0u;  // a negative scale turns the query: scores then grow with the dots
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      raw[kk] = live ? q[2 * kk] : make_uint4(0u, 0u, 0u, 0u);
      raw[kk].x ^= flip;
      raw[kk].y ^= flip;
      raw[kk].z ^= flip;
      raw[kk].w ^= flip;
    }
    qs *= query_operands<kBf16>(raw, qop, [](float v) { return max32(v); });
  }

  float m = kNoScore, M = kNoScore, l = 0.0f;
  floatx16 acc[4];  // channel 32 j + 8 (e / 4) + 4 half + e % 4 of the column
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[j][e] = 0.0f;

  Raw raw;
  if (t_begin < t_end) {
    load(t_begin, raw);
    store(buf[0], raw);
    if (t_begin + 1 < t_end) load(t_begin + 1, raw);
  }
  __syncthreads();
  for (int t = t_begin; t < t_end; ++t) {
    const Tile& x = buf[(t - t_begin) & 1];
    floatx16 s[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[tb][e] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        s[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, x.k[tb][kk][32 * half + (col ^ kk)]), qop[kk], s[tb],
                                                       0, 0, 0);
    }
    if (t + 1 < t_end) {
      store(buf[(t + 1 - t_begin) & 1], raw);
      if (t + 2 < t_end) load(t + 2, raw);
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      const int t0 = t * kTile + tb * kW;
      const float sc = fmaxf(x.ks[tb] * qs, 1e-37f), vs = x.vs[tb];  // above zero: a masked dot stays -inf
      if (t0 + kW > vis_first) {  // a token that some column of the wave does not see
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (t0 + 8 * (e >> 2) + 4 * half + (e & 3) >= vis) s[tb][e] = -__builtin_inff();
      }
      float top = s[tb][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[tb][e]);
      top = max32(top) * sc;
      const float lv = __builtin_amdgcn_logf(vs);
      // a block whose values are all zero (its scale is 1 then), or have a subnormal scale, adds to the sum alone
      bool dead = lv < -126.0f;
      if (vs == 1.0f) {
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int st = 0; st < 2; ++st) any |= or4(x.v[tb][j][st][lane]);
        dead = !__any((any & 0x7fff7fffu) != 0);
      }
      const float reach = dead ? -__builtin_inff() : top + lv;
      if (__any(top > m + kLazy || reach > M + kLazy)) {
        const float m2 = fmaxf(m, top), M2 = fmaxf(M, reach);
        l *= __builtin_amdgcn_exp2f(m - m2);
        const float f = __builtin_amdgcn_exp2f(M - M2);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] *= f;
        m = m2;
        M = M2;
      }
      const float off = dead ? -m : lv + kWeightExp - M;
      float sum = 0.0f;
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tb][e], sc, off));
        const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tb][e + 1], sc, off));
        sum += w0 + w1;
        w[e >> 1] = pack_f16(w0, w1);
      }
      l = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(fminf(-off - m, 126.0f)), l);
      if (dead) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 0u;
      }
      // step s takes tokens 8 s + 4 half + i and 16 + 8 s + 4 half + i: elements 4 s + i and 8 + 4 s + i
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const half8 wop = __builtin_bit_cast(half8, make_uint4(w[2 * st], w[2 * st + 1], w[4 + 2 * st], w[5 + 2 * st]));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, x.v[tb][j][st][lane]), wop, acc[j], 0, 0, 0);
      }
    }
    __syncthreads();
  }

  l = sum32(l);
  if (!live) return;
  if (records == 0) {
    const float f = l > 0.0f ? __builtin_amdgcn_exp2f(M - m - kWeightExp) / l : 0.0f;
    uint16_t* out = p.out + (((int64_t)b * c.Hq + hq) * p.n_max + i) * kD + 4 * half;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<uint2*>(out + 32 * j + 2 * e) = make_uint2(row_pack<kBf16>(acc[j][e] * f, acc[j][e + 1] * f),
                                                                     row_pack<kBf16>(acc[j][e + 2] * f, acc[j][e + 3] * f));
    return;
  }
  float* rec = p.ws + ((int64_t)first * c.H * p.ntile + ((int64_t)h * p.ntile + tile) * nsplit + split) * (kQ8PromptCols * (kD + 4));
  const int cc = 32 * wave + col;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<floatx4*>(rec + cc * kD + 32 * j + 2 * e + 4 * half) =
          floatx4{acc[j][e], acc[j][e + 1], acc[j][e + 2], acc[j][e + 3]};
  if (half == 0) *reinterpret_cast<floatx4*>(rec + kQ8PromptCols * kD + 4 * cc) = floatx4{M, m, l, 0.0f};
}

}  // namespace

hipError_t launch_q8_prompt(const Q8AttendArgs& a, int most, int format, int dtype, int B, hipStream_t s) {
  const dim3 grid((unsigned)(B * a.c.H * a.ntile), most), block(kThreads);
  if (format == OKVQ_Q8_INT8) {
    if (dtype == OKVQ_BF16) hipLaunchKernelGGL((k_q8_prompt<OKVQ_Q8_INT8, true>), grid, block, 0, s, a, B);
    else hipLaunchKernelGGL((k_q8_prompt<OKVQ_Q8_INT8, false>), grid, block, 0, s, a, B);
  } else {
    if (dtype == OKVQ_BF16) hipLaunchKernelGGL((k_q8_prompt<OKVQ_Q8_E4M3, true>), grid, block, 0, s, a, B);
    else hipLaunchKernelGGL((k_q8_prompt<OKVQ_Q8_E4M3, false>), grid, block, 0, s, a, B);
  }
  return hipGetLastError();
}

}  // namespace okvq
