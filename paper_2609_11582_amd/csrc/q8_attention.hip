// Attention over one layer of the paged 8-bit cache: split kernel for few rows, and the merge of its splits.
//
// A row's softmax weights are p_t = 2^(s_t - m) with s_t = q . code_t * (k_scale sm_scale log2 e), and the output is
// sum_t p_t v_scale code_t / sum_t p_t. One pass over the codes with a running m; few rows leave most of the GPU
// idle, so the sequence is split over work-groups whose partial sums a second launch joins.
//
// Split kernel. Work-group (split, KV head and tile, sequence) = 8 waves; wave w of split s takes the blocks (32
// tokens) 8 s + w, 8 (s + nsplit) + w, ... and keeps its own state for 16 query columns (the G heads of one or
// more positions), so one read of the cache serves all of them. Which blocks a wave takes does not depend on
// the sequence's length: the page table is read beside the length and not after it.
//  * Scores: 16x16x32 fp16 matrix instructions, rows = 16 tokens, columns = queries. A lane's key operand is 16
//    bytes of a token's row, widened in registers (the contraction order over channels is the lanes' own; the
//    query operand follows it). int8 codes become fp16 by a byte permute (1024 + 128 + code, exact) and one
//    subtraction, e4m3 codes by the conversion instruction: both exact.
//  * The score tile's layout (token 4 g + i, query column) is the layout of the weights as the B operand of the
//    value product (k slot 4 a + i of lane group g <-> token 16 a + 4 g + i), and the cache keeps value blocks in
//    the matching A operand order: no weight or value crosses lanes or passes through LDS.
//  * The weights enter as fp16 times the block's value scale: w = p_t v_scale 2^(m - M + 7), with M a second
//    reference, the maximum of s_t + log2 v_scale. Both references move only when a maximum passes them by 2^8,
//    so w < 2^15 keeps full precision down to 2^-21 of the largest product, whatever the blocks' scales are; the
//    sum of p_t stays in fp32, unrounded.
// Where rows see a window, or precede a tree (kSpan), a wave walks those blocks of its residue that some row of the tile sees, and masks
// their tokens row by row; a tree's part always leaves records, which q8_tree.hip joins with the drafts. One token's window of
// 1024 behind 4 sinks: 4 heads 9.6 us, 16 slots of them 9.8, one launch each (four or five blocks a wave, one after the other: latency).
// Bound: memory in large calls (131072 tokens x 4 heads 25.4 us, 5.3 TB/s), latency in small ones (32768 tokens 9.0 us: 2
// blocks a wave; 12.0 with the merge). 4 or 16 waves in place of 8 were 16 and 10 % slower on the build that took 13.4.
#include <algorithm>

#include "q8_mfma.hpp"

namespace okvq {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRecFloatsQ8 = kQ8Cols * kQ8Record;  // a split's record: [16][128] sums, then [16] of (M, m, l, 0)
static_assert(kQ8Record == kD + 4 && kWaves * kW == 256, "as the plan counts");
constexpr int kCombineRow = kD + 4;               // floats of a combine row: 16 rows of a column fall into all banks

template <int kSpan, int kFmt, bool kBf16>
__global__ __launch_bounds__(kThreads, 4) void k_q8_split(Q8AttendArgs p) {
  __shared__ __attribute__((aligned(16))) float cmb[kWaves][kQ8Cols * kCombineRow];
  __shared__ float wM[kWaves][kQ8Cols], wm[kWaves][kQ8Cols], wl[kWaves][kQ8Cols];
  const Q8View& c = p.c;
  // everything that says what there is to do, in one wait for the arguments
  const int layer = blockIdx.z;
  int ntile = p.ntile;
  Q8Order order = p.splits.order;
  uint32_t w = p.splits.part[q8_part_index(layer)], next = p.splits.part[q8_part_index(layer) + 1];
  __asm__ volatile(""
                   : "+s"(ntile), "+s"(order.split_slots), "+s"(order.slots), "+s"(order.flags), "+s"(order.most), "+s"(w), "+s"(next)
                   : "s"(c.k_codes), "s"(c.table), "s"(c.lens), "s"(c.H), "s"(c.max_pages), "s"(p.q), "s"(p.n_new), "s"(p.n_max), "s"(p.G));
  const int h = blockIdx.y / ntile, tile = blockIdx.y - h * ntile;
  const int r0 = tile * kQ8Cols;  // first row of the tile
  const int place = q8_place(order, layer, blockIdx.x);
  const Q8Part mine = q8_part(order, w, next, place, blockIdx.x, tile);
  if (mine.none) return;
  int b = place;
  const int split = mine.split, nsplit = mine.nsplit;
  if (order.flags & kQ8Reordered) b = q8_slot_at(p.splits, place);
  // tiles that may have no rows, before they load anything in advance
  if ((order.flags & kQ8Uneven) && (tile > 0 || place >= order.active_slots) && r0 >= (int64_t)uniform_load(p.n_new + b) * p.G) return;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* row = c.table + (int64_t)b * c.max_pages;
  const int stride = nsplit * kWaves;
  int block = split * kWaves + wave;

  // The query rows, column's channels 64 (kk / 2) + 16 g + 8 (kk % 2) .. + 7, of rows that may not be live
  const int i = (r0 + col) / p.G, hq = h * p.G + (r0 + col - i * p.G);
  uint4 raw[4];
  {
    const uint4* q = reinterpret_cast<const uint4*>(p.q) + (((int64_t)b * c.Hq + min(hq, c.Hq - 1)) * p.n_max + min(i, p.n_max - 1)) * 16;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) raw[kk] = q[8 * (kk >> 1) + 2 * g + (kk & 1)];
  }
  // A block's registers: key rows 16 tb + col (channels 16 g .. + 15 and 64 + 16 g .. + 15), value slots 64 j + lane,
  // and the scales, which are wave-uniform. Every address is inside the pool, so the first block is loaded before
  // the lengths say whether it is needed
  uint4 k[2][2], v[4];
  float ks, vs;
  const uint32_t ko = col * 128 + g * 16, vo = lane * 16;
  auto load_keys = [&](int64_t slot) {
    const uint8_t* at = c.k_codes + slot * kQ8Block;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      k[tb][0] = *reinterpret_cast<const uint4*>(at + (ko + tb * 2048));
      k[tb][1] = *reinterpret_cast<const uint4*>(at + (ko + tb * 2048 + 64));
    }
    ks = uniform_load(c.k_scale + slot);
  };
  auto load_values = [&](int64_t slot) {
    const uint8_t* at = c.v_codes + slot * kQ8Block;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint4*>(at + (vo + j * 1024));
    vs = uniform_load(c.v_scale + slot);
  };
  int64_t slot;
  int page;
  if constexpr (kSpan == kQ8Full) {
    slot = q8_slot(q8_page(row, block, c), h, block, c);
    load_keys(slot);
    load_values(slot);
    page = q8_page(row, block + stride, c);  // of the wave's next block
    __asm__ volatile("" ::: "memory");       // the loads above go out before the length is waited for
  }

  const int len = q8_len(c, b), n = min(max(uniform_load(p.n_new + b), 0), p.n_max);
  const int i_first = r0 / p.G, i_last = min((r0 + kQ8Cols - 1) / p.G, n - 1);
  if (i_first >= n) return;
  auto cross = [&] { return kSpan == kQ8Tree || (kSpan == kQ8Full && p.cross); };
  const int vis_first = cross() ? len : max(len - n + i_first + 1, 0);  // tokens that the first and the last row see
  const int vis_last = cross() ? len : max(len - n + i_last + 1, 0);
  const bool live = i < n;
  const int vis = live ? (cross() ? len : max(len - n + i + 1, 0)) : 0;
  const int nblk = (vis_last + kW - 1) / kW;
  // with a window the wave's blocks are numbered over those that some row of the tile sees, which the length says
  const Q8Walk walk(kSpan == kQ8Full ? 0 : p.sinks, q8_from_least<kSpan>(p, len, n, i_first), vis_last, kW);
  const int from_most = q8_from_most<kSpan>(p, len, n, i_last), end = kSpan == kQ8Full ? nblk : walk.count;
  auto real = [&](int v) { return kSpan == kQ8Full ? v : walk(v); };
  int from = 0;
  if constexpr (kSpan != kQ8Full) {
    slot = q8_slot(q8_page(row, real(block), c), h, real(block), c);
    load_keys(slot);
    load_values(slot);
    page = q8_page(row, real(block + stride), c);
    from = live ? q8_sight<kSpan>(p, b, len, n, i).from : 0;
  }

  half8 qop[4];
  float qs = p.qscale;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk)
    if (!live) raw[kk] = make_uint4(0u, 0u, 0u, 0u);
  qs *= query_operands<kBf16>(raw, qop, [](float v) { return max32(max16(v)); });

  float m = kNoScore, M = kNoScore, l = 0.0f;
  floatx4 acc[8];  // channel 16 t + 4 g + i of the column
#pragma unroll
  for (int t = 0; t < 8; ++t) acc[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  while (block < end) {
    const int t0 = real(block) * kW, next = block + stride;
    slot = q8_slot(page, h, real(next), c);
    floatx4 s[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      s[tb] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const uint4 w = k[tb][kk >> 1];
        s[tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk & 1 ? widen8<kFmt>(w.z, w.w) : widen8<kFmt>(w.x, w.y), qop[kk], s[tb], 0,
                                                       0, 0);
      }
    }
    const float sc = ks * qs;
    // the keys' registers are free: the next block's keys are on their way during the softmax and the value product,
    // its values during the next scores. Four waves on a SIMD do the rest; a second set of registers instead left
    // room for two
    if (next < end) load_keys(slot);
    float mx = -__builtin_inff();
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[tb][e] *= sc;
    // a token that some row of the tile does not see
    if (t0 + kW > vis_first || (kSpan != kQ8Full && t0 < from_most && t0 + kW > p.sinks)) {
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = t0 + 16 * tb + 4 * g + e;
          if (t >= vis || (kSpan != kQ8Full && t < from && t >= p.sinks)) s[tb][e] = -__builtin_inff();
        }
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[tb][e]);
    mx = max32(max16(mx));
    float lv = __builtin_amdgcn_logf(vs);
    // a block whose values are all zero has scale 1: it adds to the sum alone and must not move M (a subnormal
    // scale has lv = -inf here, and the same)
    if (vs == 1.0f && !__any(((or4(v[0]) | or4(v[1]) | or4(v[2]) | or4(v[3])) & 0x7f7f7f7fu) != 0)) lv = -__builtin_inff();
    if (__any(mx > m + kLazy || mx + lv > M + kLazy)) {
      const float m2 = fmaxf(m, mx), M2 = fmaxf(M, mx + lv);
      l *= __builtin_amdgcn_exp2f(m - m2);
      const float f = __builtin_amdgcn_exp2f(M - M2);
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] *= f;
      m = m2;
      M = M2;
    }
    // finite, so that a weight of zero stays zero; the bound is reached only by weights p below 2^-112
    const float f = __builtin_amdgcn_exp2f(fminf(m - M + lv + kWeightExp, 127.0f));
    uint32_t w[4];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[tb][e] - m), p1 = __builtin_amdgcn_exp2f(s[tb][e + 1] - m);
        l += p0 + p1;
        w[2 * tb + (e >> 1)] = pack_f16(p0 * f, p1 * f);
      }
    const half8 wop = __builtin_bit_cast(half8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<kFmt>(v[j].x, v[j].y), wop, acc[2 * j], 0, 0, 0);
      acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<kFmt>(v[j].z, v[j].w), wop, acc[2 * j + 1], 0, 0, 0);
    }
    if (next < end) load_values(slot);
    page = q8_page(row, real(next + stride), c);
    block = next;
  }

  // ---- combine the waves ----
  l = sum32(sum16(l));
#pragma unroll
  for (int t = 0; t < 8; ++t) *reinterpret_cast<floatx4*>(&cmb[wave][col * kCombineRow + 16 * t + 4 * g]) = acc[t];
  if (lane < kQ8Cols) {
    wM[wave][lane] = M;
    wm[wave][lane] = m;
    wl[wave][lane] = l;
  }
  __syncthreads();
  const int cc = tid >> 5, ch = (tid & 31) * 4;
  static_assert(kThreads == 32 * kQ8Cols, "32 lanes a column");
  const int ci = (r0 + cc) / p.G, chq = h * p.G + (r0 + cc - ci * p.G);
  if (ci >= n) return;
  float Mt = kNoScore, mt = kNoScore;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Mt = fmaxf(Mt, wM[w][cc]);
    mt = fmaxf(mt, wm[w][cc]);
  }
  float lt = 0.0f;
  floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    lt += wl[w][cc] * __builtin_amdgcn_exp2f(wm[w][cc] - mt);
    o += *reinterpret_cast<const floatx4*>(&cmb[w][cc * kCombineRow + ch]) * __builtin_amdgcn_exp2f(wM[w][cc] - Mt);
  }
  if (kSpan != kQ8Tree && mine.records == 0) {
    const RowFactor f(Mt, mt, lt);
    *reinterpret_cast<uint2*>(p.out + (((int64_t)b * c.Hq + chq) * p.n_max + ci) * kD + ch) =
        make_uint2(row_pack<kBf16>(f(o[0]), f(o[1])), row_pack<kBf16>(f(o[2]), f(o[3])));
    return;
  }
  int64_t at = mine.first * c.H + h * mine.records + tile * nsplit + split;
  if (kSpan == kQ8Tree && mine.records == 0) at = p.single + ((int64_t)b * c.H + h) * ntile + tile;
  float* rec = p.ws + at * kRecFloatsQ8;
  *reinterpret_cast<floatx4*>(rec + cc * kD + ch) = o;
  if ((tid & 31) == 0) *reinterpret_cast<floatx4*>(rec + kQ8Cols * kD + 4 * cc) = floatx4{Mt, mt, lt, 0.0f};
}

// Join the splits: kGroups groups of 32 lanes share a column's (a group takes every kGroups-th split, then the
// groups are added), kCols columns a work-group
template <bool kBf16, int kGroups, int kCols>
__global__ __launch_bounds__(32 * kGroups * kCols) void k_q8_merge(Q8AttendArgs p, int cols) {
  __shared__ __attribute__((aligned(16))) floatx4 part[kGroups * kCols][32];
  const int place = blockIdx.z;
  int ntile = p.ntile;
  Q8Order order = p.splits.order;
  uint32_t w = p.splits.part[place], next = p.splits.part[place + 1];
  __asm__ volatile(""  // one wait for them
                   : "+s"(ntile), "+s"(order.flags), "+s"(w), "+s"(next)
                   : "s"(p.ws), "s"(p.n_new), "s"(p.n_max), "s"(p.G), "s"(p.out), "s"(p.c.H), "s"(cols));
  const int h = blockIdx.y / ntile, tile = blockIdx.y - h * ntile;
  const int tid = threadIdx.x, lane = tid & 31, grp = (tid >> 5) % kGroups, cc = blockIdx.x * kCols + (tid >> 5) / kGroups;
  const Q8Part mine = q8_part(order, w, next, place, 0, tile);
  if (mine.records == 0) return;
  const int nsplit = mine.nsplit, b = order.flags & kQ8Reordered ? q8_slot_at(p.splits, place) : place;
  const int n = min(max(uniform_load(p.n_new + b), 0), p.n_max);
  const int r = tile * cols + cc, i = r / p.G, hq = h * p.G + (r - i * p.G);
  const bool live = i < n;
  if (kCols == 1 && !live) return;  // the whole work-group
  const int recf = cols * kQ8Record;
  const float* rec = p.ws + (int64_t)(mine.first * p.c.H + h * mine.records + tile * nsplit) * recf;
  floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  RowFactor factor(kNoScore, kNoScore, 0.0f);
  if (live) {
    // A group has 8 splits at most: their sums are on their way while the references and the softmax sum of all splits
    // are formed, which every group does for itself (a lane takes every 32nd split)
    const float* stat = rec + cols * kD + 4 * cc;
    const float* sums = rec + cc * kD + 4 * lane;
    floatx4 v[8];
    float vM[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t at = (int64_t)min(grp + k * kGroups, nsplit - 1) * recf;
      v[k] = *reinterpret_cast<const floatx4*>(sums + at);
      vM[k] = stat[at];
    }
    constexpr int kStats = (8 * kGroups + 31) / 32;
    floatx4 st[kStats];
    float M = kNoScore, m = kNoScore, l = 0.0f;
#pragma unroll
    for (int k = 0; k < kStats; ++k) {
      const int s = lane + 32 * k;
      st[k] = *reinterpret_cast<const floatx4*>(stat + (int64_t)min(s, nsplit - 1) * recf);
      if (s >= nsplit) st[k][2] = 0.0f;  // counted already
      M = fmaxf(M, st[k][0]);
      m = fmaxf(m, st[k][1]);
    }
    M = half_reduce(M, [](float a, float b) { return fmaxf(a, b); });
    m = half_reduce(m, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll
    for (int k = 0; k < kStats; ++k) l += st[k][2] * __builtin_amdgcn_exp2f(st[k][1] - m);
    l = half_reduce(l, [](float a, float b) { return a + b; });
    factor = RowFactor(M, m, l);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (grp + k * kGroups < nsplit) o += v[k] * __builtin_amdgcn_exp2f(vM[k] - M);
  }
  if constexpr (kGroups > 1) {
    part[tid >> 5][lane] = o;
    __syncthreads();
    if (grp != 0) return;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) o += part[(tid >> 5) + k][lane];
  }
  if (!live) return;
  *reinterpret_cast<uint2*>(p.out + (((int64_t)b * p.c.Hq + hq) * p.n_max + i) * kD + 4 * lane) =
      make_uint2(row_pack<kBf16>(factor(o[0]), factor(o[1])), row_pack<kBf16>(factor(o[2]), factor(o[3])));
}

}  // namespace

template <int kGroups, int kCols>
static void merge(const Q8AttendArgs& a, const Q8Plan& p, bool bf16, hipStream_t s) {
  // no work-group for columns that no row has
  const dim3 grid((p.rows + kCols - 1) / kCols, a.c.H * p.ntile, p.splits.order.split_slots), block(32 * kGroups * kCols);
  if (bf16) hipLaunchKernelGGL((k_q8_merge<true, kGroups, kCols>), grid, block, 0, s, a, p.cols);
  else hipLaunchKernelGGL((k_q8_merge<false, kGroups, kCols>), grid, block, 0, s, a, p.cols);
}

template <int kSpan>
static void split(const Q8AttendArgs& a, const Q8Plan& p, int format, bool bf16, hipStream_t s) {
  const dim3 grid(p.splits.order.most, a.c.H * p.ntile, q8_layers(p)), block(kThreads);
  if (format == OKVQ_Q8_INT8) {
    if (bf16) hipLaunchKernelGGL((k_q8_split<kSpan, OKVQ_Q8_INT8, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_q8_split<kSpan, OKVQ_Q8_INT8, false>), grid, block, 0, s, a);
  } else {
    if (bf16) hipLaunchKernelGGL((k_q8_split<kSpan, OKVQ_Q8_E4M3, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_q8_split<kSpan, OKVQ_Q8_E4M3, false>), grid, block, 0, s, a);
  }
}

hipError_t launch_q8_attention(Q8AttendArgs& a, const Q8Plan& p, int span, int format, int dtype, hipStream_t s) {
  a.ntile = p.ntile;
  a.splits = p.splits;
  const bool bf16 = dtype == OKVQ_BF16;
  hipError_t e;
  if (p.cols == kQ8WideCols) {
    e = launch_q8_wide(a, p, span, format, dtype, s);
  } else if (p.cols != kQ8Cols) {
    e = launch_q8_prompt(a, p, span, format, dtype, s);
  } else {
    if (span == kQ8Full) split<kQ8Full>(a, p, format, bf16, s);
    else if (span == kQ8Window) split<kQ8Window>(a, p, format, bf16, s);
    else split<kQ8Tree>(a, p, format, bf16, s);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  if (span == kQ8Tree) return launch_q8_tree_merge(a, p, dtype, s);
  if (p.splits.order.most == 1) return e;
  // a column to 8 groups of lanes, 16 where there are many splits (128 splits: 7.9 -> 4.5 us); 8 columns to a work-group
  // where there are few (2 splits of 32768 rows: 33 -> 8 us)
  if (p.splits.order.most > 64) merge<16, 1>(a, p, bf16, s);
  else if (p.splits.order.most > 8 || p.cols == kQ8Cols) merge<8, 1>(a, p, bf16, s);
  else merge<1, 8>(a, p, bf16, s);
  return hipGetLastError();
}

}  // namespace okvq
