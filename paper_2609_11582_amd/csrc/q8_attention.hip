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
#include <algorithm>

#include "q8_mfma.hpp"

namespace okvq {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRecFloatsQ8 = kQ8Cols * (kD + 4);  // a split's record: [16][128] sums, then [16] of (M, m, l, 0)
constexpr int kCombineRow = kD + 4;               // floats of a combine row: 16 rows of a column fall into all banks

struct BlockRegs {
  uint4 k[2][2];  // key rows 16 tb + col: channels 16 g .. + 15 and 64 + 16 g .. + 15
  uint4 v[4];     // value slots 64 j + lane
  float ks, vs;
};

template <int kFmt, bool kBf16>
__global__ __launch_bounds__(kThreads) void k_q8_split(Q8AttendArgs p) {
  __shared__ __attribute__((aligned(16))) float cmb[kWaves][kQ8Cols * kCombineRow];
  __shared__ float wM[kWaves][kQ8Cols], wm[kWaves][kQ8Cols], wl[kWaves][kQ8Cols];
  const Q8View& c = p.c;
  const int split = blockIdx.x, h = blockIdx.y / p.ntile, tile = blockIdx.y - h * p.ntile, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* row = c.table + (int64_t)b * c.max_pages;
  const int len = q8_len(c, b), n = min(max(p.n_new[b], 0), p.n_max);
  const int r0 = tile * kQ8Cols, i_first = r0 / p.G;
  if (i_first >= n) return;  // no live row in the tile
  const int i_last = min((r0 + kQ8Cols - 1) / p.G, n - 1);
  const int vis_first = p.cross ? len : max(len - n + i_first + 1, 0);  // tokens that the tile's first and last rows see
  const int vis_last = p.cross ? len : max(len - n + i_last + 1, 0);
  const int i = (r0 + col) / p.G, hq = h * p.G + (r0 + col - i * p.G);
  const bool live = i < n;
  const int vis = live ? (p.cross ? len : max(len - n + i + 1, 0)) : 0;
  const int nblk = (vis_last + kW - 1) / kW, stride = p.nsplit * kWaves;

  auto load = [&](int block, BlockRegs& x) {
    const int64_t slot = q8_slot(q8_page(row, block, c), h, block, c);
    const uint4* k = reinterpret_cast<const uint4*>(c.k_codes + slot * kQ8Block) + col * 8 + g;
    const uint4* v = reinterpret_cast<const uint4*>(c.v_codes + slot * kQ8Block) + lane;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      x.k[tb][0] = k[tb * 128];
      x.k[tb][1] = k[tb * 128 + 4];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x.v[j] = v[64 * j];
    x.ks = c.k_scale[slot];
    x.vs = c.v_scale[slot];
  };

  // query operands: column's channels 64 (kk / 2) + 16 g + 8 (kk % 2) .. + 7
  half8 qop[4];
  float qs = p.qscale;
  {
    const uint4* q = reinterpret_cast<const uint4*>(p.q) + (((int64_t)b * c.Hq + hq) * p.n_max + i) * 16;
    uint4 raw[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) raw[kk] = live ? q[8 * (kk >> 1) + 2 * g + (kk & 1)] : make_uint4(0u, 0u, 0u, 0u);
    qs *= query_operands<kBf16>(raw, qop, [](float v) { return max32(max16(v)); });
  }

  float m = kNoScore, M = kNoScore, l = 0.0f;
  floatx4 acc[8];  // channel 16 t + 4 g + i of the column
#pragma unroll
  for (int t = 0; t < 8; ++t) acc[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  auto compute = [&](int block, const BlockRegs& x) {
    const int t0 = block * kW;
    floatx4 s[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      s[tb] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const uint4 w = x.k[tb][kk >> 1];
        s[tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk & 1 ? widen8<kFmt>(w.z, w.w) : widen8<kFmt>(w.x, w.y), qop[kk], s[tb], 0,
                                                       0, 0);
      }
    }
    const float sc = x.ks * qs;
    float mx = -__builtin_inff();
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[tb][e] *= sc;
    if (t0 + kW > vis_first) {  // a token that some row of the tile does not see
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + 16 * tb + 4 * g + e >= vis) s[tb][e] = -__builtin_inff();
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[tb][e]);
    mx = max32(max16(mx));
    float lv = __builtin_amdgcn_logf(x.vs);
    // a block whose values are all zero has scale 1: it adds to the sum alone and must not move M (a subnormal
    // scale has lv = -inf here, and the same)
    if (x.vs == 1.0f && !__any(((or4(x.v[0]) | or4(x.v[1]) | or4(x.v[2]) | or4(x.v[3])) & 0x7f7f7f7fu) != 0)) lv = -__builtin_inff();
    if (__any(mx > m + kLazy || mx + lv > M + kLazy)) {
      const float m2 = fmaxf(m, mx), M2 = fmaxf(M, mx + lv);
      l *= __builtin_amdgcn_exp2f(m - m2);
      const float f = __builtin_amdgcn_exp2f(M - M2);
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] *= f;
      m = m2;
      M = M2;
    }
    const float f = __builtin_amdgcn_exp2f(fminf(m - M + lv + kWeightExp, 100.0f));
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
      acc[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<kFmt>(x.v[j].x, x.v[j].y), wop, acc[2 * j], 0, 0, 0);
      acc[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<kFmt>(x.v[j].z, x.v[j].w), wop, acc[2 * j + 1], 0, 0, 0);
    }
  };

  // two register sets: the next block's loads are in flight while one is computed
  BlockRegs xa, xb;
  int block = split * kWaves + wave;
  if (block < nblk) load(block, xa);
  while (block < nblk) {
    if (block + stride < nblk) load(block + stride, xb);
    compute(block, xa);
    block += stride;
    if (block >= nblk) break;
    if (block + stride < nblk) load(block + stride, xa);
    compute(block, xb);
    block += stride;
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
  if (p.nsplit == 1) {
    const float f = lt > 0.0f ? __builtin_amdgcn_exp2f(Mt - mt - kWeightExp) / lt : 0.0f;
    *reinterpret_cast<uint2*>(p.out + (((int64_t)b * c.Hq + chq) * p.n_max + ci) * kD + ch) =
        make_uint2(row_pack<kBf16>(o[0] * f, o[1] * f), row_pack<kBf16>(o[2] * f, o[3] * f));
    return;
  }
  float* rec = p.ws + (((int64_t)b * gridDim.y + blockIdx.y) * p.nsplit + split) * kRecFloatsQ8;
  *reinterpret_cast<floatx4*>(rec + cc * kD + ch) = o;
  if ((tid & 31) == 0) *reinterpret_cast<floatx4*>(rec + kQ8Cols * kD + 4 * cc) = floatx4{Mt, mt, lt, 0.0f};
}

// Join the splits of one column: 8 groups of 32 lanes take every eighth split, then the groups are added.
template <bool kBf16>
__global__ __launch_bounds__(256) void k_q8_merge(Q8AttendArgs p, int cols) {
  __shared__ float factor[kQ8MaxSplits];
  __shared__ __attribute__((aligned(16))) floatx4 part[8][32];
  __shared__ float scale;
  const int cc = blockIdx.x, h = blockIdx.y / p.ntile, tile = blockIdx.y - h * p.ntile, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63;
  const int n = min(max(p.n_new[b], 0), p.n_max);
  const int r = tile * cols + cc, i = r / p.G, hq = h * p.G + (r - i * p.G);
  if (i >= n) return;
  const int recf = cols * (kD + 4);
  const float* rec = p.ws + ((int64_t)b * gridDim.y + blockIdx.y) * p.nsplit * recf;
  if (tid < 64) {
    float M = kNoScore, m = kNoScore, l = 0.0f;
    float fM[kQ8MaxSplits / 64];
#pragma unroll
    for (int k = 0; k < kQ8MaxSplits / 64; ++k) {
      const int s = lane + 64 * k;
      floatx4 st = {kNoScore, kNoScore, 0.0f, 0.0f};
      if (s < p.nsplit) st = *reinterpret_cast<const floatx4*>(rec + (int64_t)s * recf + cols * kD + 4 * cc);
      fM[k] = st[0];
      const float m2 = fmaxf(m, st[1]);
      l = l * __builtin_amdgcn_exp2f(m - m2) + st[2] * __builtin_amdgcn_exp2f(st[1] - m2);
      m = m2;
      M = fmaxf(M, st[0]);
    }
    M = wave_max(M);
    const float mt = wave_max(m);
    l *= __builtin_amdgcn_exp2f(m - mt);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
#pragma unroll
    for (int k = 0; k < kQ8MaxSplits / 64; ++k) factor[lane + 64 * k] = __builtin_amdgcn_exp2f(fM[k] - M);
    if (lane == 0) scale = l > 0.0f ? __builtin_amdgcn_exp2f(M - mt - kWeightExp) / l : 0.0f;
  }
  __syncthreads();
  const int grp = tid >> 5, ch = (tid & 31) * 4;
  floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = grp; s < p.nsplit; s += 8) o += *reinterpret_cast<const floatx4*>(rec + (int64_t)s * recf + cc * kD + ch) * factor[s];
  part[grp][tid & 31] = o;
  __syncthreads();
  if (tid >= 32) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) o += part[k][tid];
  o *= scale;
  *reinterpret_cast<uint2*>(p.out + (((int64_t)b * p.c.Hq + hq) * p.n_max + i) * kD + ch) =
      make_uint2(row_pack<kBf16>(o[0], o[1]), row_pack<kBf16>(o[2], o[3]));
}

}  // namespace

Q8Plan q8_plan(int B, int H, int G, int n_max, int max_len) {
  Q8Plan p;
  const int64_t rows = (int64_t)n_max * G;
  p.cols = rows <= kQ8Cols ? kQ8Cols : kQ8PromptCols;
  p.ntile = (int)((rows + p.cols - 1) / p.cols);
  const int64_t units = (int64_t)B * H * p.ntile;
  int64_t want, most;
  if (p.cols == kQ8Cols) {
    // work-groups for every compute unit; a split has at least a block for each wave
    want = (kQ8Groups + units - 1) / units;
    most = ((max_len + kW - 1) / kW + kWaves - 1) / kWaves;
  } else {
    want = (kQ8PromptGroups + units - 1) / units;
    most = (max_len + kQ8PromptSplit - 1) / kQ8PromptSplit;
  }
  p.nsplit = (int)std::max<int64_t>(1, std::min({want, most, (int64_t)kQ8MaxSplits}));
  return p;
}

size_t q8_plan_bytes(const Q8Plan& p, int B, int H) {
  if (p.nsplit == 1) return 0;
  return (size_t)B * H * p.ntile * p.nsplit * p.cols * (kD + 4) * sizeof(float);
}

// A call of u units (tiles of every sequence and head) has at most the groups it is split into and u records more;
// calls of fewer rows have no more units of the same kind, and a call of few rows has B H
size_t q8_workspace_bound(int B, int H, int G, int n_max, int max_len) {
  const size_t few = ((size_t)B * H + kQ8Groups) * kQ8Cols;
  const int64_t rows = (int64_t)n_max * G;
  size_t many = 0;
  if (rows > kQ8Cols) {
    const size_t units = (size_t)B * H * ((rows + kQ8PromptCols - 1) / kQ8PromptCols);
    many = std::min(units, (size_t)kQ8PromptGroups) + kQ8PromptGroups;  // units of kQ8PromptGroups and more are not split
    many *= kQ8PromptCols;
  }
  (void)max_len;
  return std::max(few, many) * (kD + 4) * sizeof(float);
}

hipError_t launch_q8_attention(Q8AttendArgs a, const Q8Plan& p, int format, int dtype, int B, hipStream_t s) {
  a.nsplit = p.nsplit;
  a.ntile = p.ntile;
  const dim3 grid(p.nsplit, a.c.H * p.ntile, B), block(kThreads);
  const bool bf16 = dtype == OKVQ_BF16;
  hipError_t e;
  if (p.cols == kQ8PromptCols) {
    e = launch_q8_prompt(a, format, dtype, B, s);
  } else if (format == OKVQ_Q8_INT8) {
    if (bf16) hipLaunchKernelGGL((k_q8_split<OKVQ_Q8_INT8, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_q8_split<OKVQ_Q8_INT8, false>), grid, block, 0, s, a);
  } else {
    if (bf16) hipLaunchKernelGGL((k_q8_split<OKVQ_Q8_E4M3, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_q8_split<OKVQ_Q8_E4M3, false>), grid, block, 0, s, a);
  }
  if (p.cols == kQ8Cols) e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const dim3 mgrid(p.cols, a.c.H * p.ntile, B);
  if (bf16) hipLaunchKernelGGL((k_q8_merge<true>), mgrid, dim3(256), 0, s, a, p.cols);
  else hipLaunchKernelGGL((k_q8_merge<false>), mgrid, dim3(256), 0, s, a, p.cols);
  return hipGetLastError();
}

}  // namespace okvq
