// Attention of drafted trees, the drafts' part: joins the splits of the cache's part with it.
//
// A row's softmax runs over the cache's tokens and the drafts that its mask names (its ancestors and itself, a few). The
// split, wide and prompt kernels leave records (M, m, l, sums) of the cache's part (q8_attention.hip); here a work-group takes 1 to 8
// query columns, attends their drafts in fp32 from their rows as they are, with a running maximum, and adds all parts: as a
// record the drafts' part has m, l and sums 2^-8 p v, whose reference M is m + kWeightExp + 8 (256 values of bfloat16's
// largest size stay finite).
//
// Bound: latency. A column's splits and drafts are dealt to kGroups groups of 32 lanes (4 channels a lane), drafts by their number,
// so that a group meets few of them, four at a time; the splits' statistics and sums are loaded first and used last. 112 columns x 4
// heads, 32 splits 4.8 us. With few splits a group takes a column alone, 8 columns a work-group (8 slots of up to 175 columns x 4 heads,
// 4 splits: 6.9 us, with 8 groups a column 16.8).
#include "q8_mfma.hpp"

namespace okvq {
namespace {

constexpr float kDraftExp = 8.0f;  // drafts of a call: 2^8 at most
constexpr int kAhead = 4;          // drafts whose rows are on their way together

template <bool kBf16, int kGroups, int kCols>
__global__ __launch_bounds__(32 * kGroups * kCols) void k_q8_tree_merge(Q8AttendArgs p, int cols) {
  constexpr int kTeams = kGroups * kCols;
  __shared__ __attribute__((aligned(16))) floatx4 part[kTeams][32];
  __shared__ float gm[kTeams], gl[kTeams];
  static_assert(32 % kGroups == 0, "a word of a mask is dealt to the groups evenly");
  const int place = blockIdx.z;
  int ntile = p.ntile;
  Q8Order order = p.splits.order;
  uint32_t w = p.splits.part[q8_part_index(place)], next = p.splits.part[q8_part_index(place) + 1];
  __asm__ volatile(""  // one wait for them
                   : "+s"(ntile), "+s"(order.split_slots), "+s"(order.slots), "+s"(order.flags), "+s"(w), "+s"(next)
                   : "s"(p.ws), "s"(p.n_new), "s"(p.n_max), "s"(p.G), "s"(p.out), "s"(p.c.H), "s"(cols), "s"(p.visible), "s"(p.words),
                     "s"(p.kd), "s"(p.vd), "s"(p.q));
  const int h = blockIdx.y / ntile, tile = blockIdx.y - h * ntile;
  const Q8Part mine = q8_part(order, w, next, place, 0, tile);
  const int b = order.flags & kQ8Reordered ? q8_slot_at(p.splits, place) : place;
  const int tid = threadIdx.x, lane = tid & 31, team = tid >> 5, grp = team % kGroups, cc = blockIdx.x * kCols + team / kGroups;
  const int r = tile * cols + min(cc, cols - 1), i = r / p.G, hq = h * p.G + (r - i * p.G);
  const int row = min(i, p.n_max - 1);  // of teams without one: any

  // the splits' sums, a group every kGroups-th, and their statistics, a lane every 32nd. These and the rows below go out before the
  // count says whether they are needed (every column of a tile has its place in a record)
  const int nsplit = mine.nsplit, recf = cols * kQ8Record;
  const int64_t first = mine.records ? (int64_t)(mine.first * p.c.H + h * mine.records + tile * nsplit)
                                     : p.single + ((int64_t)b * p.c.H + h) * ntile + tile;
  const int at_col = r - tile * cols;
  const float* rec = p.ws + first * recf;
  const float* stat = rec + cols * kD + 4 * at_col;
  const float* sums = rec + at_col * kD + 4 * lane;
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
#pragma unroll
  for (int k = 0; k < kStats; ++k) st[k] = *reinterpret_cast<const floatx4*>(stat + (int64_t)min(lane + 32 * k, nsplit - 1) * recf);

  // the group's drafts: those of its residue modulo kGroups
  const uint32_t* mask = p.visible + ((int64_t)b * p.n_max + row) * p.words;
  uint32_t word = mask[0];
  const uint2 qr = *reinterpret_cast<const uint2*>(p.q + (((int64_t)b * p.c.Hq + min(hq, p.c.Hq - 1)) * p.n_max + row) * kD + 4 * lane);
  __asm__ volatile("" ::: "memory");
  const int n = min(max(uniform_load(p.n_new + b), 0), p.n_max);
  if ((tile * cols + (int)blockIdx.x * kCols) / p.G >= n) return;  // the whole work-group
  const bool live = cc < cols && i < n;
  if (kGroups == 1 && !live) return;
  const float q0 = row_lo<kBf16>(qr.x), q1 = row_hi<kBf16>(qr.x), q2 = row_lo<kBf16>(qr.y), q3 = row_hi<kBf16>(qr.y);
  const int64_t rows = ((int64_t)b * p.c.H + h) * p.n_max * kD + 4 * lane;
  uint32_t mine_of_word = 0;
#pragma unroll
  for (int k = 0; k < 32; k += kGroups) mine_of_word |= 1u << k;
  mine_of_word <<= grp;
  float dm = kNoScore, dl = 0.0f;
  floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int at_word = 0; 32 * at_word < n; ++at_word) {
    uint32_t bits = live ? q8_named(word, at_word, n) & mine_of_word : 0u;
    if (32 * (at_word + 1) < n) word = mask[at_word + 1];
    while (bits) {
      uint2 kr[kAhead], vr[kAhead];
      bool named[kAhead];
      int j = 0;
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        named[a] = bits != 0;
        if (named[a]) j = 32 * at_word + __builtin_ctz(bits);  // else the draft before it once more, without weight
        bits &= bits - 1;
        kr[a] = *reinterpret_cast<const uint2*>(p.kd + rows + (int64_t)j * kD);
        vr[a] = *reinterpret_cast<const uint2*>(p.vd + rows + (int64_t)j * kD);
      }
      float s[kAhead], top = dm;
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        s[a] = q0 * row_lo<kBf16>(kr[a].x);
        s[a] = __builtin_fmaf(q1, row_hi<kBf16>(kr[a].x), s[a]);
        s[a] = __builtin_fmaf(q2, row_lo<kBf16>(kr[a].y), s[a]);
        s[a] = __builtin_fmaf(q3, row_hi<kBf16>(kr[a].y), s[a]);
        s[a] = half_reduce(s[a], [](float a, float b) { return a + b; }) * p.qscale;
        if (!named[a]) s[a] = -__builtin_inff();
        top = fmaxf(top, s[a]);
      }
      const float f = __builtin_amdgcn_exp2f(dm - top);
      dl *= f;
      o *= f;
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const float e = __builtin_amdgcn_exp2f(s[a] - top), ev = e * 0x1p-8f;
        dl += e;
        o[0] = __builtin_fmaf(ev, row_lo<kBf16>(vr[a].x), o[0]);
        o[1] = __builtin_fmaf(ev, row_hi<kBf16>(vr[a].x), o[1]);
        o[2] = __builtin_fmaf(ev, row_lo<kBf16>(vr[a].y), o[2]);
        o[3] = __builtin_fmaf(ev, row_hi<kBf16>(vr[a].y), o[3]);
      }
      dm = top;
    }
  }
  if constexpr (kGroups > 1) {
    if (lane == 0) {
      gm[team] = dm;
      gl[team] = dl;
    }
    __syncthreads();
  }

  // references and softmax sum of all parts, which every group forms for itself
  float M = kNoScore, m = kNoScore, l = 0.0f;
#pragma unroll
  for (int k = 0; k < kStats; ++k) {
    if (lane + 32 * k >= nsplit) st[k][2] = 0.0f;  // counted already
    M = fmaxf(M, st[k][0]);
    m = fmaxf(m, st[k][1]);
  }
  M = half_reduce(M, [](float a, float b) { return fmaxf(a, b); });
  m = half_reduce(m, [](float a, float b) { return fmaxf(a, b); });
  float um[kGroups], ul[kGroups];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    um[g] = kGroups > 1 ? gm[team - grp + g] : dm;
    ul[g] = kGroups > 1 ? gl[team - grp + g] : dl;
    m = fmaxf(m, um[g]);
    M = fmaxf(M, um[g] + (kWeightExp + kDraftExp));
  }
#pragma unroll
  for (int k = 0; k < kStats; ++k) l += st[k][2] * __builtin_amdgcn_exp2f(st[k][1] - m);
  l = half_reduce(l, [](float a, float b) { return a + b; });
#pragma unroll
  for (int g = 0; g < kGroups; ++g) l += ul[g] * __builtin_amdgcn_exp2f(um[g] - m);
  o *= __builtin_amdgcn_exp2f(dm + (kWeightExp + kDraftExp) - M);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (grp + k * kGroups < nsplit) o += v[k] * __builtin_amdgcn_exp2f(vM[k] - M);
  if constexpr (kGroups > 1) {
    part[team][lane] = o;
    __syncthreads();
    if (grp != 0) return;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) o += part[team + k][lane];
  }
  if (!live) return;
  const RowFactor factor(M, m, l);
  *reinterpret_cast<uint2*>(p.out + (((int64_t)b * p.c.Hq + hq) * p.n_max + i) * kD + 4 * lane) =
      make_uint2(row_pack<kBf16>(factor(o[0]), factor(o[1])), row_pack<kBf16>(factor(o[2]), factor(o[3])));
}

template <int kGroups, int kCols>
void merge(const Q8AttendArgs& a, const Q8Plan& p, bool bf16, hipStream_t s) {
  const dim3 grid((p.rows + kCols - 1) / kCols, a.c.H * p.ntile, p.splits.order.slots), block(32 * kGroups * kCols);
  if (bf16) hipLaunchKernelGGL((k_q8_tree_merge<true, kGroups, kCols>), grid, block, 0, s, a, p.cols);
  else hipLaunchKernelGGL((k_q8_tree_merge<false, kGroups, kCols>), grid, block, 0, s, a, p.cols);
}

}  // namespace

hipError_t launch_q8_tree_merge(const Q8AttendArgs& a, const Q8Plan& p, int dtype, hipStream_t s) {
  static_assert(kQ8MaxSplits == 16 * 8, "a group takes 8 splits at most");
  switch (q8_tree_merge(p).groups) {
    case 16: merge<16, 1>(a, p, dtype == OKVQ_BF16, s); break;
    case 8: merge<8, 1>(a, p, dtype == OKVQ_BF16, s); break;
    case 4: merge<4, 2>(a, p, dtype == OKVQ_BF16, s); break;
    case 2: merge<2, 4>(a, p, dtype == OKVQ_BF16, s); break;
    default: merge<1, 8>(a, p, dtype == OKVQ_BF16, s);
  }
  return hipGetLastError();
}

}  // namespace okvq
