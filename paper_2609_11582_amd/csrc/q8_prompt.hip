// Attention of many rows over the paged 8-bit cache: chunks and whole prompts.
//
// The formulas are the split kernel's (q8_attention.hip); here the products dominate: 4 x 128 flops a row and token,
// far above what the 256 bytes of a token cost. A work-group takes 256 query columns (the G heads of consecutive
// positions), 8 waves of 32 (or 128 and 4, where those fill the GPU better), and walks the tokens in tiles of 64:
//  * Codes are widened to fp16 once a tile and work-group, on their way from memory through registers to LDS (two
//    buffers: the next tile is written while one is used, the one after is in flight). Both kinds lie in LDS as
//    the 32x32x16 matrix instructions' A operands, 1 KB each, so every read is 64 lanes x 16 contiguous bytes.
//  * Scores: rows = 32 tokens, columns = queries, the query held in registers. A lane holds half the tokens of one
//    column, so the softmax is in-lane but for one exchange of maxima; the weights are the value product's B operand
//    as they stand (k slot of step s, half h, 4 a + i <-> token 16 a + 8 s + 4 h + i, which is also the order of 8
//    consecutive bytes of a value block).
//  * The weights are formed in one fused step as 2^(dot * scale + c), c = log2 v_scale + 7 - M; their sum, divided
//    by the block's factor, is the block's share of the softmax sum.
//  * Where rows see a window, or precede a tree (kSpan), the walk is over the blocks that some row of the work-group sees: a wave's
//    products stop at the last tile that its own rows see, and it goes on bringing tiles for the others in a loop of its own (a
//    branch around the products in one loop costs 60 to 160 spilled registers: 410 us in place of 190). 8192 rows
//    x 28 heads with windows of 1024: 175 us, 0.64 PFLOP/s of what the rows see (1024 + 128 / 7 + 63 tokens are computed for each),
//    with 2.0 us a pass of 64 tokens, 5.8 before the first and 2.4 after the last of a work-group's 19.
// Bound: issue and power together. 512 rows against 4 x 65536 tokens run at 1.0 PFLOP/s (a large bf16 product of the
// library at 1.2). Under the counters (1184 us, 1.88 GHz) the matrix cores are busy 47 % and the vector units 55 % of the SIMD
// cycles, the LDS 31 %.
#include <algorithm>

#include "q8_mfma.hpp"

namespace okvq {
namespace {

constexpr int kTile = 64;                 // tokens
constexpr int kOperand = 64;              // 16-byte slots of a matrix operand
constexpr float kLeastWeight = -60.0f;    // log2 of the weight at the reference m; at most 2^(kLazy - 60), zero as fp16

template <int kPieces>
struct Raw {                              // a thread's 16 bytes of keys or of values of kPieces blocks, the blocks' scales,
  uint4 x[kPieces];                       // and which blocks of which pages are next
  float scale[kPieces];
  int block[kPieces], page[kPieces];
};

template <int kSpan, int kFmt, bool kBf16, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void k_q8_prompt(Q8AttendArgs p, int width) {
  constexpr int kCols = 32 * kWaves, kPieces = 8 / kWaves;
  // two buffers of keys [block][16 channels][half h, token: at token ^ (channels & 7)] and of values
  // [block][32 channels][step s][half h, channel], as operands; the scales of three tiles, as the keys are ahead
  __shared__ uint4 kbuf[2][2][8][kOperand], vbuf[2][2][4][2][kOperand];
  __shared__ float kscale[3][2], vscale[2][2];
  const Q8View& c = p.c;
  Q8Order order = p.splits.order;
  int ntile = p.ntile;
  __asm__ volatile(""  // one wait for the arguments
                   : "+s"(order.split_slots), "+s"(order.active_slots), "+s"(order.slots), "+s"(order.flags), "+s"(ntile)
                   : "s"(c.k_codes), "s"(c.table), "s"(c.lens), "s"(c.max_pages), "s"(p.n_new), "s"(p.n_max), "s"(p.G), "s"(c.H));
  const Q8Tile at = q8_tile(order, c.H, ntile, width, blockIdx.x, blockIdx.y);
  if (at.place < 0) return;
  const int tile = at.tile, h = at.h;
  Q8Part mine;
  if (at.place < order.split_slots) mine = q8_part(order, p.splits.part[at.place], p.splits.part[at.place + 1], at.place, blockIdx.y, tile);
  else mine.none = false;
  if (mine.none) return;
  const int b = order.flags & kQ8Reordered ? q8_slot_at(p.splits, at.place) : at.place, split = mine.split, nsplit = mine.nsplit;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* table = c.table + (int64_t)b * c.max_pages;
  const int len = q8_len(c, b), n = min(max(uniform_load(p.n_new + b), 0), p.n_max);
  const int r0 = tile * kCols, i_first = r0 / p.G;
  if (i_first >= n) return;
  const int i_last = min((r0 + kCols - 1) / p.G, n - 1);
  auto cross = [&] { return kSpan == kQ8Tree || (kSpan == kQ8Full && p.cross); };
  const int vis_last = cross() ? len : max(len - n + i_last + 1, 0);
  // the wave's columns, and the tokens that they see
  const int r = r0 + 32 * wave + col, i = r / p.G, hq = h * p.G + (r - i * p.G);
  const bool live = i < n;
  const int vis = live ? (cross() ? len : max(len - n + i + 1, 0)) : 0;
  const int wave_first = (r0 + 32 * wave) / p.G;
  const int vis_first = wave_first >= n ? 0 : cross() ? len : max(len - n + wave_first + 1, 0);
  const bool busy = wave_first < n;  // a wave without a live column has only its part of the tiles to bring
  // with a window the blocks are numbered over those that some row of the work-group sees, and a tile is two in a row of these
  const Q8Walk walk(kSpan == kQ8Full ? 0 : p.sinks, q8_from_least<kSpan>(p, len, n, i_first), vis_last, kW);
  const int steps = kSpan == kQ8Full ? (vis_last + kTile - 1) / kTile : (walk.count + 1) / 2;
  // what the wave's rows see at most, and where the last of them begins
  const int wave_last = min((r0 + 32 * wave + 31) / p.G, n - 1);
  const int vis_most = cross() ? len : max(len - n + wave_last + 1, 0);
  const int from_most = q8_from_most<kSpan>(p, len, n, wave_last);
  const int from = kSpan != kQ8Full && live ? q8_sight<kSpan>(p, b, len, n, i).from : 0;
  const int per = (steps + nsplit - 1) / nsplit, t_begin = min(split * per, steps), t_end = min(t_begin + per, steps);

  // Staging: a thread has 16 bytes of key row tid / 8 % 32 and of value slot tid % 256 of kPieces of the tile's two blocks.
  // Behind the sequence its last block stands for those to come: what a zero weight multiplies has to be finite. Values
  // of a subnormal scale count as zero, as their logarithm is none.
  // Page ids and scales come through the scalar cache, whose waits are waits for all LDS reads too: a page is fetched a
  // tile before its codes, and what is fetched is waited for at the head of the loop, where nothing is in flight.
  const int sb = kPieces == 2 ? 0 : wave >> 2, krow = (tid >> 3) & 31, kchunk = tid & 7, vslot = tid & 255;
  const int last = max((len - 1) / kW, 0);
  auto fetch_page = [&](int t, Raw<kPieces>& r) {
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      r.block[e] = min(kSpan == kQ8Full ? 2 * t + sb + e : walk(2 * t + sb + e), last);
      r.page[e] = uniform_load(table + min(r.block[e] >> c.bshift, c.max_pages - 1));
    }
  };
  auto load = [&](const uint8_t* codes, const float* scales, Raw<kPieces>& r) {
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      const int64_t slot = q8_slot(min(max(r.page[e], 0), c.P - 1), h, r.block[e], c);
      r.x[e] = *reinterpret_cast<const uint4*>(codes + slot * kQ8Block + vslot * 16);
      r.scale[e] = uniform_load(scales + slot);
    }
  };
  // codes of tile t, whose page is known, and the page of the tile after it
  auto load_keys = [&](int t, Raw<kPieces>& r) {
    load(c.k_codes, c.k_scale, r);
    fetch_page(t + 1, r);
  };
  auto load_values = [&](int t, Raw<kPieces>& r) {
    load(c.v_codes, c.v_scale, r);
    fetch_page(t + 1, r);
  };
  auto fetched = [&](const Raw<kPieces>& r) {
#pragma unroll
    for (int e = 0; e < kPieces; ++e) __asm__ volatile("" ::"s"(r.page[e]), "s"(r.scale[e]));
  };
  auto store_keys = [&](int u, const Raw<kPieces>& r) {
    const int kp = krow ^ kchunk;
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      uint4* to = kbuf[u & 1][sb + e][kchunk];
      to[kp] = __builtin_bit_cast(uint4, widen8<kFmt>(r.x[e].x, r.x[e].y));
      to[32 + kp] = __builtin_bit_cast(uint4, widen8<kFmt>(r.x[e].z, r.x[e].w));
      kscale[u % 3][sb + e] = r.scale[e];  // every lane writes the same
    }
  };
  auto store_values = [&](int u, const Raw<kPieces>& r) {
    const int j = vslot >> 6, g = (vslot >> 4) & 3, ch = vslot & 15;
#pragma unroll
    for (int e = 0; e < kPieces; ++e) {
      uint4* to = vbuf[u & 1][sb + e][j][g >> 1] + 32 * (g & 1) + ch;
      const uint32_t keep = r.scale[e] >= 0x1p-126f ? ~0u : 0u;
      to[0] = __builtin_bit_cast(uint4, widen8<kFmt>(r.x[e].x & keep, r.x[e].y & keep));
      to[16] = __builtin_bit_cast(uint4, widen8<kFmt>(r.x[e].z & keep, r.x[e].w & keep));
      vscale[u & 1][sb + e] = keep ? r.scale[e] : 1.0f;
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

  // The loop runs the next tile's scores beside this tile's softmax: matrix and vector instructions of one wave overlap
  // where they do not depend on each other. So the keys in LDS are a tile ahead of the values.
  const int nt = t_end - t_begin;
  Raw<kPieces> kr, vr;
  floatx16 s[2], s2[2];
  float top[2] = {kNoScore, kNoScore};  // largest dot of each block of s
  auto scores = [&](const uint4 (&k)[2][8][kOperand], floatx16 (&d)[2]) {
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) d[tb][e] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        d[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, k[tb][kk][32 * half + (col ^ kk)]), qop[kk], d[tb], 0,
                                                       0, 0);
    }
  };
  auto tops = [&](const floatx16 (&d)[2]) {
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      float x = d[tb][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) x = fmaxf(x, d[tb][e]);
      top[tb] = max32(x);
    }
  };
  if (nt > 0) {
    fetch_page(t_begin, kr);
    fetch_page(t_begin, vr);
    load_keys(t_begin, kr);
    load_values(t_begin, vr);
    store_keys(0, kr);
    store_values(0, vr);
    load_keys(t_begin + 1, kr);
    load_values(t_begin + 1, vr);
    store_keys(1, kr);
    load_keys(t_begin + 2, kr);
    __syncthreads();
    if (busy) {
      scores(kbuf[0], s);
      tops(s);
    }
    __syncthreads();  // the first pass of the loop overwrites that buffer
  }
  auto stage = [&](int u) {
    store_values(u + 1, vr);
    store_keys(u + 2, kr);
    load_values(t_begin + u + 2, vr);
    load_keys(t_begin + u + 3, kr);
  };
  // with a window a wave stops at the last tile that its rows see, and only stages those for other waves' rows
  int u = 0, own = nt;
  if constexpr (kSpan != kQ8Full) own = busy ? min(max((walk.before(vis_most, kW) + 1) / 2 - t_begin, 0), nt) : 0;
  for (; u < own; ++u) {
    fetched(kr);
    fetched(vr);
    if (kSpan == kQ8Full && !busy) {
      stage(u);
      __syncthreads();
      continue;
    }
    const int cur = u & 1;
    if constexpr (kSpan == kQ8Full) {
      const int t0 = (t_begin + u) * kTile;
      if (t0 + kTile > vis_first) {  // a token that some column of the wave does not see
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (t0 + tb * kW + 8 * (e >> 2) + 4 * half + (e & 3) >= vis) s[tb][e] = -__builtin_inff();
        tops(s);
      }
    } else {
      const int base[2] = {walk(2 * (t_begin + u)) * kW, walk(2 * (t_begin + u) + 1) * kW};
      bool edge = false;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        const int t0 = base[tb], vis_at = vis - t0 - 4 * half, from_at = from - t0 - 4 * half;
        if (t0 + kW > vis_first) {
          edge = true;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (8 * (e >> 2) + (e & 3) >= vis_at) s[tb][e] = -__builtin_inff();
        }
        if (t0 < from_most && t0 + kW > p.sinks) {
          edge = true;
          const int sinks_at = p.sinks - t0 - 4 * half;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (8 * (e >> 2) + (e & 3) < from_at && 8 * (e >> 2) + (e & 3) >= sinks_at) s[tb][e] = -__builtin_inff();
        }
      }
      if (edge) tops(s);
    }
    float sc[2], lv[2], high[2], reach[2], off[2], gain[2];
    bool dead[2] = {false, false};
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      sc[tb] = fmaxf(kscale[u % 3][tb] * qs, 1e-37f);  // above zero: a masked dot stays -inf
      lv[tb] = __builtin_amdgcn_logf(vscale[cur][tb]);
    }
    if (vscale[cur][0] == 1.0f || vscale[cur][1] == 1.0f) {
      // a block whose values are all zero (its scale is 1 then) adds to the sum alone and must not move M
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int st = 0; st < 2; ++st) any |= or4(vbuf[cur][tb][j][st][lane]);
        dead[tb] = !__any((any & 0x7fff7fffu) != 0);
      }
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      high[tb] = top[tb] * sc[tb];
      reach[tb] = dead[tb] ? -__builtin_inff() : high[tb] + lv[tb];
    }
    const float high2 = fmaxf(high[0], high[1]), reach2 = fmaxf(reach[0], reach[1]);
    if (__any(high2 > m + kLazy || reach2 > M + kLazy)) {
      const float m2 = fmaxf(m, high2), M2 = fmaxf(M, reach2);
      l *= __builtin_amdgcn_exp2f(m - m2);
      const float f = __builtin_amdgcn_exp2f(M - M2);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] *= f;
      m = m2;
      M = M2;
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      // zero codes take any finite weight. Values too small beside others for a weight in fp16 take one that is zero
      // there and still adds to the sum in fp32 (without it, scales 2^110 apart lost their blocks' part of the sum)
      off[tb] = dead[tb] ? -m : fmaxf(lv[tb] + kWeightExp - M, kLeastWeight - m);
      gain[tb] = __builtin_amdgcn_exp2f(-off[tb] - m);
    }
    // One stretch without a branch: the next scores beside this tile's weights, then the value product beside the next
    // scores' maxima and the tiles to come on their way to LDS (behind the last tile they are some page's, and unused)
    scores(kbuf[cur ^ 1], s2);
    uint32_t w[2][8];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tb][e], sc[tb], off[tb]));
        const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tb][e + 1], sc[tb], off[tb]));
        sum += w0 + w1;
        w[tb][e >> 1] = pack_f16(w0, w1);
      }
      l = __builtin_fmaf(sum, gain[tb], l);
    }
    stage(u);
    // step st takes tokens 8 st + 4 half + i and 16 + 8 st + 4 half + i: elements 4 st + i and 8 + 4 st + i
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const half8 wop = __builtin_bit_cast(half8, make_uint4(w[tb][2 * st], w[tb][2 * st + 1], w[tb][4 + 2 * st], w[tb][5 + 2 * st]));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, vbuf[cur][tb][j][st][lane]), wop, acc[j], 0, 0, 0);
      }
    s[0] = s2[0];
    s[1] = s2[1];
    tops(s);
    __syncthreads();
  }
  if constexpr (kSpan != kQ8Full)
    for (; u < nt; ++u) {
      fetched(kr);
      fetched(vr);
      stage(u);
      __syncthreads();
    }

  l = sum32(l);
  if (!live) return;
  if (kSpan != kQ8Tree && mine.records == 0) {
    const RowFactor f(M, m, l);
    uint16_t* out = p.out + (((int64_t)b * c.Hq + hq) * p.n_max + i) * kD + 4 * half;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<uint2*>(out + 32 * j + 2 * e) = make_uint2(row_pack<kBf16>(f(acc[j][e]), f(acc[j][e + 1])),
                                                                     row_pack<kBf16>(f(acc[j][e + 2]), f(acc[j][e + 3])));
    return;
  }
  int64_t place = mine.first * c.H + h * mine.records + tile * nsplit + split;
  if (kSpan == kQ8Tree && mine.records == 0) place = p.single + ((int64_t)b * c.H + h) * ntile + tile;
  float* rec = p.ws + place * (kCols * kQ8Record);
  const int cc = 32 * wave + col;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<floatx4*>(rec + cc * kD + 32 * j + 2 * e + 4 * half) =
          floatx4{acc[j][e], acc[j][e + 1], acc[j][e + 2], acc[j][e + 3]};
  if (half == 0) *reinterpret_cast<floatx4*>(rec + kCols * kD + 4 * cc) = floatx4{M, m, l, 0.0f};
}

}  // namespace

template <int kSpan, int kFmt, bool kBf16>
static void launch(const Q8AttendArgs& a, const Q8Plan& p, hipStream_t s) {
  const int width = q8_layers(p) * a.c.H * p.ntile;
  const dim3 grid((unsigned)width, p.splits.order.most);
  if (p.cols == 256) hipLaunchKernelGGL((k_q8_prompt<kSpan, kFmt, kBf16, 8>), grid, dim3(512), 0, s, a, width);
  else hipLaunchKernelGGL((k_q8_prompt<kSpan, kFmt, kBf16, 4>), grid, dim3(256), 0, s, a, width);
}

template <int kSpan>
static void launch(const Q8AttendArgs& a, const Q8Plan& p, int format, bool bf16, hipStream_t s) {
  if (format == OKVQ_Q8_INT8) bf16 ? launch<kSpan, OKVQ_Q8_INT8, true>(a, p, s) : launch<kSpan, OKVQ_Q8_INT8, false>(a, p, s);
  else bf16 ? launch<kSpan, OKVQ_Q8_E4M3, true>(a, p, s) : launch<kSpan, OKVQ_Q8_E4M3, false>(a, p, s);
}

hipError_t launch_q8_prompt(const Q8AttendArgs& a, const Q8Plan& p, int span, int format, int dtype, hipStream_t s) {
  if (span == kQ8Full) launch<kQ8Full>(a, p, format, dtype == OKVQ_BF16, s);
  else if (span == kQ8Window) launch<kQ8Window>(a, p, format, dtype == OKVQ_BF16, s);
  else launch<kQ8Tree>(a, p, format, dtype == OKVQ_BF16, s);
  return hipGetLastError();
}

}  // namespace okvq
