// Attention of some dozens of query columns over the paged 8-bit cache, where rows see a window or precede a tree of drafts:
// between the split kernel (q8_attention.hip), which reads and widens the codes once for 16 columns, and the prompt kernel
// (q8_prompt.hip), which computes 256 whatever there are.
//
// The formulas are the prompt kernel's: weights 2^(dot * scale + off) with off = log2 v_scale + 7 - M, whose sum, divided by the
// block's factor, is the block's share of the softmax sum. Work-group = 8 waves and 64 columns of a head; wave w of split s
// walks the blocks (32 tokens) 8 s + w, 8 (s + nsplit) + w, ... that some row sees. Codes go from memory through registers, widened
// there, straight into the matrix instructions (32x32x16, two tiles of 32 columns); no barrier in the loop.
//  * The columns' sums are 128 registers. The query operands do not fit beside them: they lie in LDS (16 KB) and are read for
//    every block, 1 KB for each matrix instruction of the scores.
//  * Keys enter as their codes, widened exactly: an offset on int8's, taken off again behind the product, would put a score's error at
//    2^-24 of 128 scale |sum q| in place of scale sum |q code|, 10 times the error that the other kernels' roundings allow at
//    queries of mean 20 against blocks with one channel of 1000.
//  * The work-groups are numbered through, those of a slot, head and split side by side on one XCD, so that its L2 serves the
//    tiles that read the same codes, and no XCD has more of them than others (a ragged batch launched as slots x splits
//    put 33 on some XCDs' 32 compute units, which took a second round: 62 us for 8 slots of 133 to 175 columns).
//  * At the end the waves' sums, brought to one reference, go through LDS 32 columns x 64 channels a round, in two buffers.
// Bound: latency in short calls: 112 columns x 4 heads against 32768 tokens 19.3 us, of which the loop (4 blocks a wave) is 8, start and
// end are 3.9 and 3.5; 8 ragged slots of up to 175 columns x 4 heads at up to 8192 tokens 27 us. In long ones issue: 512 columns x 4
// heads against 131072 tokens 158 us, 0.87 PFLOP/s, of which 149 are 128 blocks of each SIMD's two waves: a block of 32 tokens x 64 columns
// takes 1.16 us with int8, 1.08 with e4m3 (from calls of 32768 tokens, 53 and 50 us with their merge, and of 131072, 165 and 153). There the
// vector units are busy 66 % and the matrix cores 39 % of the SIMD cycles, the LDS 11 % of the compute units', at 2.1 GHz.
#include "q8_mfma.hpp"

namespace okvq {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kTiles = kQ8WideCols / 32;
constexpr int kHalfRow = kD / 2 + 4;           // floats of a combine row: 8 rows fall into all banks
constexpr float kLeastWeight = -60.0f;         // log2 of the weight at the reference m, as in the prompt kernel

struct WideShared {
  union {
    uint4 qop[8][kTiles][64];                                    // contraction step, columns, lane
    float cmb[2][kWaves][32 * kHalfRow];
  };
  float wM[kWaves][kQ8WideCols], wm[kWaves][kQ8WideCols], wl[kWaves][kQ8WideCols];
  floatx4 total[kQ8WideCols];                                    // (M, m, l, 0) of all waves
  float qscale[kQ8WideCols];
  int vis[kQ8WideCols], from[kQ8WideCols];                       // what a column's row sees
};

template <int kSpan, int kFmt, bool kBf16>
__global__ __launch_bounds__(kThreads, 2) void k_q8_wide(Q8AttendArgs p, Q8Units units) {
  __shared__ __attribute__((aligned(16))) char shared[sizeof(WideShared)];
  WideShared& sh = *reinterpret_cast<WideShared*>(shared);
  const Q8View& c = p.c;
  int ntile = p.ntile;
  __asm__ volatile(""  // one wait for the arguments
                   : "+s"(ntile)
                   : "s"(c.k_codes), "s"(c.v_codes), "s"(c.k_scale), "s"(c.v_scale), "s"(c.table), "s"(c.lens), "s"(c.H), "s"(c.Hq), "s"(c.P),
                     "s"(c.max_pages), "s"(c.bshift), "s"(p.q), "s"(p.n_new), "s"(p.n_max), "s"(p.G), "s"(p.window), "s"(p.sinks),
                     "s"(p.splits.order.split_slots), "s"(p.splits.order.flags), "s"(p.splits.part[0]), "s"(units.split), "s"(units.per));
  const Q8Unit mine = q8_unit(p.splits, units, c.H, ntile, blockIdx.x);
  if (mine.place < 0) return;
  const int h = mine.h, tile = mine.tile, nsplit = mine.nsplit;
  const int b = p.splits.order.flags & kQ8Reordered ? q8_slot_at(p.splits, mine.place) : mine.place;
  const int r0 = tile * kQ8WideCols;  // first row of the tile
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* row = c.table + (int64_t)b * c.max_pages;
  const int stride = nsplit * kWaves;
  int block = mine.split * kWaves + wave;

  // A block's registers: of key row col the channels 32 e + 16 half .. + 15; of the values, operands of step st: 8 tokens of channel
  // 32 j + col; and the scales, which are wave-uniform. Every address is inside the pool
  uint4 k[4];
  uint2 v[4][2];
  float ks, vs;
  const uint32_t ko = col * 128 + half * 16, vo = half * 256 + (col & 15) * 16 + (col >> 4) * 8;
  auto load_keys = [&](int64_t slot) {
    const uint8_t* at = c.k_codes + slot * kQ8Block;
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = *reinterpret_cast<const uint4*>(at + (ko + e * 32));
    ks = uniform_load(c.k_scale + slot);
  };
  auto load_values = [&](int64_t slot) {
    const uint8_t* at = c.v_codes + slot * kQ8Block;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int st = 0; st < 2; ++st) v[j][st] = *reinterpret_cast<const uint2*>(at + (vo + j * 1024 + st * 512));
    vs = uniform_load(c.v_scale + slot);
  };
  // the query rows, 8 lanes a column, which hold channels 16 part .. + 15; of rows that may not be live
  const int qcol = 8 * wave + (lane >> 3), part = lane & 7, qi = (r0 + qcol) / p.G, hq = h * p.G + (r0 + qcol - qi * p.G);
  uint4 raw[2];
  {
    const uint4* q = reinterpret_cast<const uint4*>(p.q) + (((int64_t)b * c.Hq + min(hq, c.Hq - 1)) * p.n_max + min(qi, p.n_max - 1)) * 16 + 2 * part;
    raw[0] = q[0];
    raw[1] = q[1];
  }
  int64_t slot;
  int page;
  // without a window the first blocks are known before the length says whether they are needed
  const bool whole = kSpan == kQ8Tree && p.window == INT32_MAX;
  if (whole) {
    slot = q8_slot(q8_page(row, block, c), h, block, c);
    load_keys(slot);
    load_values(slot);
    page = q8_page(row, block + stride, c);
    __asm__ volatile("" ::: "memory");  // the loads above go out before the length is waited for
  }
  const int len = q8_len(c, b), n = min(max(uniform_load(p.n_new + b), 0), p.n_max);
  const int i_first = r0 / p.G, i_last = min((r0 + kQ8WideCols - 1) / p.G, n - 1);
  if (i_first >= n) return;
  // what the rows of the tile see, and the blocks that this leaves
  const int vis_first = kSpan == kQ8Tree ? len : max(len - n + i_first + 1, 0);
  const int vis_last = kSpan == kQ8Tree ? len : max(len - n + i_last + 1, 0);
  const Q8Walk walk(p.sinks, q8_from_least<kSpan>(p, len, n, i_first), vis_last, kW);
  const int from_most = q8_from_most<kSpan>(p, len, n, i_last), end = walk.count;
  if (!whole) {
    slot = q8_slot(q8_page(row, walk(block), c), h, walk(block), c);
    load_keys(slot);
    load_values(slot);
    page = q8_page(row, walk(block + stride), c);  // of the wave's next block
  }

  {  // the query operands
    const bool live = qi < n;
    const uint32_t flip = p.qscale < 0.0f ? 0x80008000u : 0u;  // a negative scale turns the query: scores then grow with the dots
    half8 op[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      raw[e].x = live ? raw[e].x ^ flip : 0u;
      raw[e].y = live ? raw[e].y ^ flip : 0u;
      raw[e].z = live ? raw[e].z ^ flip : 0u;
      raw[e].w = live ? raw[e].w ^ flip : 0u;
    }
    const float f = query_operands<kBf16>(raw, op, [](float x) {
      x = fmaxf(x, fdpp<0xB1>(x));
      x = fmaxf(x, fdpp<0x4E>(x));
      return fmaxf(x, fswap4(x));
    });
    // step 2 (part / 2) + e, lanes of half part % 2
#pragma unroll
    for (int e = 0; e < 2; ++e) sh.qop[2 * (part >> 1) + e][qcol >> 5][32 * (part & 1) + (qcol & 31)] = __builtin_bit_cast(uint4, op[e]);
    if (part == 0) {
      const Q8Sight sight = live ? q8_sight<kSpan>(p, b, len, n, qi) : Q8Sight{0, 0};
      sh.vis[qcol] = sight.end;
      sh.from[qcol] = sight.from;
      sh.qscale[qcol] = fabsf(p.qscale) * f;
    }
  }
  __syncthreads();

  float m[kTiles], M[kTiles], l[kTiles], qs[kTiles];
  floatx16 acc[kTiles][4];  // channel 32 j + 8 (e / 4) + 4 half + e % 4 of the column
#pragma unroll
  for (int ct = 0; ct < kTiles; ++ct) {
    m[ct] = M[ct] = kNoScore;
    l[ct] = 0.0f;
    qs[ct] = sh.qscale[32 * ct + col];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[ct][j][e] = 0.0f;
  }

  // The two waves of a SIMD lead in turn: left alone the older one ends a third of its blocks earlier, and the younger one's last
  // blocks run without a partner (8 slots of up to 25 drafts 34.4 -> 33.8 us)
  int turn = wave >> 2;
  while (block < end) {
    if ((turn ^= 1) == 0) __builtin_amdgcn_s_setprio(1);
    else __builtin_amdgcn_s_setprio(0);
    __asm__ volatile("" ::: "memory");  // the query operands stay in LDS
    const int t0 = walk(block) * kW, next = block + stride;
    slot = q8_slot(page, h, walk(next), c);
    floatx16 s[kTiles];
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[ct][e] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint4 w = k[kk >> 1];
      const half8 key = kk & 1 ? widen8<kFmt>(w.z, w.w) : widen8<kFmt>(w.x, w.y);
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct)
        s[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key, __builtin_bit_cast(half8, sh.qop[kk][ct][lane]), s[ct], 0, 0, 0);
    }
    const float scale = ks;
    // the keys' registers are free: the next block's keys are on their way during the softmax and the value product, its values
    // during the next scores
    if (next < end) load_keys(slot);
    if (t0 + kW > vis_first || (t0 < from_most && t0 + kW > p.sinks)) {  // a token that some row of the tile does not see
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct) {
        const int vis_at = sh.vis[32 * ct + col] - t0 - 4 * half, from_at = sh.from[32 * ct + col] - t0 - 4 * half;
        const int sinks_at = p.sinks - t0 - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = 8 * (e >> 2) + (e & 3);
          if (at >= vis_at || (at < from_at && at >= sinks_at)) s[ct][e] = -__builtin_inff();
        }
      }
    }
    // a block whose values are all zero (its scale is 1 then) adds to the sum alone and must not move M; so does one of a
    // subnormal scale, whose logarithm is none and whose values count as zero
    const float lv = __builtin_amdgcn_logf(vs);
    bool dead = false;
    if (vs < 0x1p-126f) {
      dead = true;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j][0] = v[j][1] = make_uint2(0u, 0u);
    } else if (vs == 1.0f) {
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) any |= v[j][0].x | v[j][0].y | v[j][1].x | v[j][1].y;
      dead = !__any((any & 0x7f7f7f7fu) != 0);
    }
    float sc[kTiles], high[kTiles], reach[kTiles];
    bool moves = false;
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct) {
      float x = s[ct][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) x = fmaxf(x, s[ct][e]);
      sc[ct] = fmaxf(scale * qs[ct], 1e-37f);  // above zero: a masked dot stays -inf
      high[ct] = max32(x) * sc[ct];
      reach[ct] = dead ? -__builtin_inff() : high[ct] + lv;
      moves |= high[ct] > m[ct] + kLazy || reach[ct] > M[ct] + kLazy;
    }
    if (__any(moves)) {
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct) {
        const bool moved = high[ct] > m[ct] + kLazy || reach[ct] > M[ct] + kLazy;
        const float m2 = moved ? fmaxf(m[ct], high[ct]) : m[ct], M2 = moved ? fmaxf(M[ct], reach[ct]) : M[ct];
        l[ct] *= __builtin_amdgcn_exp2f(m[ct] - m2);
        const float f = __builtin_amdgcn_exp2f(M[ct] - M2);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[ct][j] *= f;
        m[ct] = m2;
        M[ct] = M2;
      }
    }
    uint32_t w[kTiles][8];
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct) {
      // zero codes take any finite weight. Values too small beside others for a weight in fp16 take one that is zero there and
      // still adds to the sum in fp32
      const float off = dead ? -m[ct] : fmaxf(lv + kWeightExp - M[ct], kLeastWeight - m[ct]);
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ct][e], sc[ct], off));
        const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ct][e + 1], sc[ct], off));
        sum += w0 + w1;
        w[ct][e >> 1] = pack_f16(w0, w1);
      }
      l[ct] = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(-off - m[ct]), l[ct]);
    }
    // step st takes tokens 8 st + 4 half + i and 16 + 8 st + 4 half + i: elements 4 st + i and 8 + 4 st + i
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const half8 value = widen8<kFmt>(v[j][st].x, v[j][st].y);
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          const half8 wop = __builtin_bit_cast(half8, make_uint4(w[ct][2 * st], w[ct][2 * st + 1], w[ct][4 + 2 * st], w[ct][5 + 2 * st]));
          acc[ct][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, wop, acc[ct][j], 0, 0, 0);
        }
      }
    if (next < end) load_values(slot);
    page = q8_page(row, walk(next + stride), c);
    block = next;
  }

  __builtin_amdgcn_s_setprio(0);

  // ---- combine the waves ----
#pragma unroll
  for (int ct = 0; ct < kTiles; ++ct) {
    l[ct] = sum32(l[ct]);
    if (half == 0) {
      sh.wM[wave][32 * ct + col] = M[ct];
      sh.wm[wave][32 * ct + col] = m[ct];
      sh.wl[wave][32 * ct + col] = l[ct];
    }
  }
  __syncthreads();  // and no wave reads query operands any more
  if (tid < kQ8WideCols) {
    float Mt = kNoScore, mt = kNoScore, lt = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      Mt = fmaxf(Mt, sh.wM[w][tid]);
      mt = fmaxf(mt, sh.wm[w][tid]);
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) lt += sh.wl[w][tid] * __builtin_amdgcn_exp2f(sh.wm[w][tid] - mt);
    sh.total[tid] = floatx4{Mt, mt, lt, 0.0f};
  }
  const bool direct = kSpan != kQ8Tree && mine.records == 0;
  int64_t at = mine.first * c.H + h * mine.records + tile * nsplit + mine.split;
  if (kSpan == kQ8Tree && mine.records == 0) at = p.single + ((int64_t)b * c.H + h) * ntile + tile;
  float* rec = p.ws + at * (kQ8WideCols * kQ8Record);
  const int cc = tid >> 4, ch = (tid & 15) * 4;
  static_assert(kThreads == 16 * 32, "16 lanes a column");
#pragma unroll
  for (int ct = 0; ct < kTiles; ++ct) {
    if ((r0 + 32 * ct) / p.G >= n) return;  // no row from here on
    float Mt = kNoScore;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) Mt = fmaxf(Mt, sh.wM[w][32 * ct + col]);
    const float f = __builtin_amdgcn_exp2f(M[ct] - Mt);
    const int cl = 32 * ct + cc, ci = (r0 + cl) / p.G, chq = h * p.G + (r0 + cl - ci * p.G);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float* mine_at = &sh.cmb[r][wave][col * kHalfRow + 4 * half];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const floatx16& a = acc[ct][2 * r + (e >> 2)];
        const int i = 4 * (e & 3);
        *reinterpret_cast<floatx4*>(mine_at + 8 * e) = floatx4{a[i], a[i + 1], a[i + 2], a[i + 3]} * f;
      }
      __syncthreads();
      floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) o += *reinterpret_cast<const floatx4*>(&sh.cmb[r][w][cc * kHalfRow + ch]);
      if (ci >= n) continue;
      if (direct) {
        const floatx4 t = sh.total[cl];
        const RowFactor factor(t[0], t[1], t[2]);
        *reinterpret_cast<uint2*>(p.out + (((int64_t)b * c.Hq + chq) * p.n_max + ci) * kD + 64 * r + ch) =
            make_uint2(row_pack<kBf16>(factor(o[0]), factor(o[1])), row_pack<kBf16>(factor(o[2]), factor(o[3])));
      } else {
        *reinterpret_cast<floatx4*>(rec + cl * kD + 64 * r + ch) = o;
        if (r == 0 && (tid & 15) == 0) *reinterpret_cast<floatx4*>(rec + kQ8WideCols * kD + 4 * cl) = sh.total[cl];
      }
    }
  }
}

template <int kSpan>
void launch(const Q8AttendArgs& a, const Q8Plan& p, int format, bool bf16, hipStream_t s) {
  const Q8Units units = q8_units(p, a.c.H);
  const dim3 grid((unsigned)q8_wide_groups(p, a.c.H)), block(kThreads);
  if (format == OKVQ_Q8_INT8) {
    if (bf16) hipLaunchKernelGGL((k_q8_wide<kSpan, OKVQ_Q8_INT8, true>), grid, block, 0, s, a, units);
    else hipLaunchKernelGGL((k_q8_wide<kSpan, OKVQ_Q8_INT8, false>), grid, block, 0, s, a, units);
  } else {
    if (bf16) hipLaunchKernelGGL((k_q8_wide<kSpan, OKVQ_Q8_E4M3, true>), grid, block, 0, s, a, units);
    else hipLaunchKernelGGL((k_q8_wide<kSpan, OKVQ_Q8_E4M3, false>), grid, block, 0, s, a, units);
  }
}

}  // namespace

hipError_t launch_q8_wide(const Q8AttendArgs& a, const Q8Plan& p, int span, int format, int dtype, hipStream_t s) {
  if (span == kQ8Window) launch<kQ8Window>(a, p, format, dtype == OKVQ_BF16, s);
  else launch<kQ8Tree>(a, p, format, dtype == OKVQ_BF16, s);
  return hipGetLastError();
}

}  // namespace okvq
