// Head norms and rotary positions in one pass, and their gradient.
//
// A row x of 128 channels becomes R (w * x * r) with r = 1 / sqrt(mean(x^2) + eps) and R the rotation of its pairs
// (rotary.hip: angles as 64-bit fractions of a turn). With dy the gradient of the row that came out and g = R^T dy:
//   dx = r (w g - x r^2 mean(w g x)),   dw = sum over rows of g x r.
// All in fp32, each row rounded once; the row's sums go through the 8 lanes that carry it.
//
// Bound: memory (one read and one write of every row; two reads and one write backwards): 32768 tokens x 32 heads 100 us, 5.3
// TB/s (a large copy 5.17); backwards, with the weights' sum, 8192 tokens x 32 heads 47 us, 4 sequences of up to 2999 tokens x 18
// heads 35 us, of which the sum and its launch are 7 to 9. One token is bound by its launch (3.5 us, 12 a call). The split is the rotation's: a
// work-group takes T tokens, whose sines and cosines go to LDS once; a lane keeps those of its 8 pairs, times the
// weights, in registers for all heads of a kind; eight lanes carry a row, 32 bytes each way.
//
// The weights' gradient: a lane adds up its 16 channels over all the rows that it meets, a work-group its lanes, and
// a last launch the work-groups, all in a fixed order: the same inputs give the same bits. So the backward's
// work-groups are few (kNormParts: one round of the GPU; 8192 tokens x 32 heads, inputs in the last-level cache, 38.5 us, with 1024
// 40.4, 512 37.6, but 4 sequences of 2999 x 18 heads 29.7, 29.7 and 30.3) and take one tile after the other. Batches of more than
// 256 sequences take a launch for each 256, which all use the same work-groups' sums: later ones add to what is there.
#include <algorithm>

#include "q8.hpp"
#include "wave_ops.hpp"

namespace okvq {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Cosine and sine of the pairs of tokens t0 .. t0 + nt - 1 of sequence b
template <int T>
__device__ __forceinline__ void angles(float2 (&cs)[T][64], const RotaryArgs& p, int b, int t0, int nt, int tid) {
  for (int i = tid; i < nt * 64; i += kThreads) {
    const int pair = i & 63;
    const int64_t pos = p.pos[((int64_t)b * 3 + p.axis[pair]) * p.n + t0 + (i >> 6)];
    const int32_t frac = (int32_t)(((uint64_t)pos * p.turn[pair]) >> 32);  // turns in units of 2^-32, signed
    float s, c;
    sincospif((float)frac * 0x1p-31f, &s, &c);
    cs[i >> 6][pair] = make_float2(c, s);
  }
}

// Lane j of a row's 8 holds channels 8 j .. + 7 as values 0 .. 7 and 64 + 8 j .. + 7 as 8 .. 15; its pair e of 8 is
// values (e, 8 + e), or (2 e, 2 e + 1) of neighbours
template <bool kAdjacent>
__host__ __device__ constexpr int first_of(int e) {
  return kAdjacent ? 2 * e : e;
}
template <bool kAdjacent>
__host__ __device__ constexpr int second_of(int e) {
  return kAdjacent ? 2 * e + 1 : e + 8;
}
template <bool kAdjacent>
__device__ __forceinline__ void lane_angles(const float2 (&cs)[64], int j, float (&co)[8], float (&si)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int pair = kAdjacent ? 4 * j + 2 * (e & 1) + 32 * (e >> 1) : 8 * j + 2 * e;
    const float4 r = *reinterpret_cast<const float4*>(&cs[pair]);
    co[2 * e] = r.x;
    si[2 * e] = r.y;
    co[2 * e + 1] = r.z;
    si[2 * e + 1] = r.w;
  }
}
__device__ __forceinline__ void lane_weights(const float* w, int j, float (&x)[16]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 r = *reinterpret_cast<const float4*>(w + 8 * j + 4 * (e & 1) + 64 * (e >> 1));
    x[4 * e] = r.x;
    x[4 * e + 1] = r.y;
    x[4 * e + 2] = r.z;
    x[4 * e + 3] = r.w;
  }
}
template <bool kBf16>
__device__ __forceinline__ void unpack(const uint4 (&raw)[2], float (&x)[16]) {
  const uint32_t u[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    x[2 * d] = row_lo<kBf16>(u[d]);
    x[2 * d + 1] = row_hi<kBf16>(u[d]);
  }
}
template <bool kBf16>
__device__ __forceinline__ void store(uint16_t* at, const float (&y)[16]) {
  uint32_t u[8];
#pragma unroll
  for (int d = 0; d < 8; ++d) u[d] = row_pack<kBf16>(y[2 * d], y[2 * d + 1]);
  *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
  *reinterpret_cast<uint4*>(at + 64) = make_uint4(u[4], u[5], u[6], u[7]);
}
__device__ __forceinline__ void load(const uint16_t* at, uint4 (&raw)[2]) {
  raw[0] = *reinterpret_cast<const uint4*>(at);
  raw[1] = *reinterpret_cast<const uint4*>(at + 64);
}
// over the 8 lanes of a row
__device__ __forceinline__ float row_sum(float v) {
  v += fdpp<0xB1>(v);
  v += fdpp<0x4E>(v);
  return v + fswap4(v);
}
__device__ __forceinline__ float inverse_rms(const float (&x)[16], float eps) {
  float ss = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
  return __builtin_amdgcn_rsqf(row_sum(ss) * (1.0f / kD) + eps);
}
// first of a lane's heads h0, h0 + kStep, ... that is one of the keys', which follow hq of the queries'
template <int kStep>
__device__ __forceinline__ int first_key(int h0, int hq) {
  return h0 + max((hq - h0 + kStep - 1) / kStep, 0) * kStep;
}
// a lane's 16 bytes of each half of a row
__device__ __forceinline__ uint16_t* place(const okvq_rows& r, int b, int h, int t, int j) {
  return static_cast<uint16_t*>(r.data) + (int64_t)b * r.batch_stride + h * r.head_stride + (int64_t)t * r.token_stride + 8 * j;
}

template <bool kBf16, bool kAdjacent, int T>
__global__ __launch_bounds__(kThreads) void k_norm_rotary(NormRotaryArgs a, int ntile) {
  __shared__ __attribute__((aligned(16))) float2 cs[T][64];
  constexpr int kHeads = 8 / T, kStep = kWaves * kHeads;  // heads of a wave at once, of the work-group
  constexpr int kRows = T == 8 ? 2 : 4;                   // rows that a lane loads at once
  const RotaryArgs& p = a.r;
  const int tid = threadIdx.x, lane = tid & 63, heads = p.hq + p.hk;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 7, t = (lane >> 3) % T, h0 = wave * kHeads + (lane >> 3) / T;
  for (int64_t unit = blockIdx.x; unit < (int64_t)ntile * p.nb; unit += gridDim.x) {
    const int bi = (int)(unit / ntile), t0 = (int)(unit % ntile) * T, b = p.b0 + bi;
    const int nt = min(p.lens.lens[bi] - t0, T);
    if (nt <= 0) continue;
    angles<T>(cs, p, b, t0, nt, tid);
    __syncthreads();
    if (t < nt) {
      float co[8], si[8];
      lane_angles<kAdjacent>(cs[t], j, co, si);
      auto rows = [&](const okvq_rows& in, const okvq_rows& out, const float* weight, int h, int from, int to) {
        if (h >= to) return;
        float w[16], c1[8], s1[8], c2[8], s2[8];  // cosine and sine times the weight of a pair's first and second value
        lane_weights(weight, j, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c1[e] = co[e] * w[first_of<kAdjacent>(e)];
          s1[e] = si[e] * w[first_of<kAdjacent>(e)];
          c2[e] = co[e] * w[second_of<kAdjacent>(e)];
          s2[e] = si[e] * w[second_of<kAdjacent>(e)];
        }
        for (; h < to; h += kRows * kStep) {
          uint4 raw[kRows][2];
#pragma unroll
          for (int i = 0; i < kRows; ++i) load(place(in, b, min(h + i * kStep, to - 1) - from, t0 + t, j), raw[i]);
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            if (h + i * kStep >= to) break;
            float x[16], y[16];
            unpack<kBf16>(raw[i], x);
            const float r = inverse_rms(x, a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x1 = x[first_of<kAdjacent>(e)] * r, x2 = x[second_of<kAdjacent>(e)] * r;
              y[first_of<kAdjacent>(e)] = __builtin_fmaf(x1, c1[e], -(x2 * s2[e]));
              y[second_of<kAdjacent>(e)] = __builtin_fmaf(x2, c2[e], x1 * s1[e]);
            }
            store<kBf16>(place(out, b, h + i * kStep - from, t0 + t, j), y);
          }
        }
      };
      rows(p.q, p.q_out, a.q_weight, h0, 0, p.hq);
      rows(p.k, p.k_out, a.k_weight, first_key<kStep>(h0, p.hq), p.hq, heads);
    }
    __syncthreads();  // the next unit overwrites the table
  }
}

// Rows of gradients, and the work-group's part of the weights' [q, k][128] at a.parts + 256 work-group: added to what an earlier
// launch left there in the first `kept` of them, stored in the others
template <bool kBf16, bool kAdjacent, int T>
__global__ __launch_bounds__(kThreads) void k_norm_rotary_grad(NormRotaryArgs a, int ntile, int kept) {
  __shared__ __attribute__((aligned(16))) float2 cs[T][64];
  __shared__ float sums[kWaves][2 * kD];
  constexpr int kHeads = 8 / T, kStep = kWaves * kHeads, kGradRows = T == 4 ? 1 : 2;
  const RotaryArgs& p = a.r;
  const int tid = threadIdx.x, lane = tid & 63, heads = p.hq + p.hk;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 7, t = (lane >> 3) % T, h0 = wave * kHeads + (lane >> 3) / T;
  float dw[2][16] = {};
  for (int64_t unit = blockIdx.x; unit < (int64_t)ntile * p.nb; unit += gridDim.x) {
    const int bi = (int)(unit / ntile), t0 = (int)(unit % ntile) * T, b = p.b0 + bi;
    const int nt = min(p.lens.lens[bi] - t0, T);
    if (nt <= 0) continue;
    angles<T>(cs, p, b, t0, nt, tid);
    __syncthreads();
    if (t < nt) {
      float co[8], si[8];
      lane_angles<kAdjacent>(cs[t], j, co, si);
      auto rows = [&](const okvq_rows& in, const okvq_rows& grad, const okvq_rows& out, const float* weight, int h, int from,
                      int to, float (&sum)[16]) {
        if (h >= to) return;
        float w[16];
        lane_weights(weight, j, w);
        for (; h < to; h += kGradRows * kStep) {
          uint4 raw[kGradRows][2], draw[kGradRows][2];
#pragma unroll
          for (int i = 0; i < kGradRows; ++i) {
            const int head = min(h + i * kStep, to - 1) - from;
            load(place(in, b, head, t0 + t, j), raw[i]);
            load(place(grad, b, head, t0 + t, j), draw[i]);
          }
#pragma unroll
          for (int i = 0; i < kGradRows; ++i) {
            if (h + i * kStep >= to) break;
            float x[16], dy[16], g[16], dx[16];
            unpack<kBf16>(raw[i], x);
            unpack<kBf16>(draw[i], dy);
            const float r = inverse_rms(x, a.eps);
            float dot = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int u = first_of<kAdjacent>(e), v = second_of<kAdjacent>(e);
              g[u] = __builtin_fmaf(dy[u], co[e], dy[v] * si[e]);
              g[v] = __builtin_fmaf(dy[v], co[e], -(dy[u] * si[e]));
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              x[e] *= r;
              sum[e] = __builtin_fmaf(g[e], x[e], sum[e]);
              g[e] *= w[e];
              dot = __builtin_fmaf(g[e], x[e], dot);
            }
            dot = row_sum(dot) * (1.0f / kD);
#pragma unroll
            for (int e = 0; e < 16; ++e) dx[e] = r * __builtin_fmaf(-x[e], dot, g[e]);
            store<kBf16>(place(out, b, h + i * kStep - from, t0 + t, j), dx);
          }
        }
      };
      rows(p.q, a.q_grad, p.q_out, a.q_weight, h0, 0, p.hq, dw[0]);
      rows(p.k, a.k_grad, p.k_out, a.k_weight, first_key<kStep>(h0, p.hq), p.hq, heads, dw[1]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int kind = 0; kind < 2; ++kind)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = dw[kind][e];  // over the wave's lanes with the same channels
      v += fswap8(v);
      v = sum32(sum16(v));
      if (lane < 8) sums[wave][kind * kD + 8 * j + (e & 7) + 64 * (e >> 3)] = v;
    }
  __syncthreads();
  float v = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v += sums[w][tid];
  static_assert(kThreads == 2 * kD, "a thread for each weight");
  float* at = a.parts + (int64_t)blockIdx.x * (2 * kD) + tid;
  *at = (int)blockIdx.x < kept ? *at + v : v;
}

// The parts' sum: a work-group takes 16 weights, 64 threads each, which hold 64 bits
constexpr int kSumCols = 16, kSumRows = 64;
__global__ __launch_bounds__(kSumCols* kSumRows) void k_norm_weight_sum(const float* parts, int n, float* dq_weight, float* dk_weight) {
  __shared__ double s[kSumRows][kSumCols];
  const int tid = threadIdx.x, c = tid % kSumCols, r = tid / kSumCols, at = blockIdx.x * kSumCols + c;
  double v = 0.0;
#pragma unroll 8
  for (int i = r; i < n; i += kSumRows) v += (double)parts[(int64_t)i * (2 * kD) + at];
  s[r][c] = v;
  __syncthreads();
  if (r != 0) return;
  v = 0.0;
#pragma unroll 8
  for (int i = 0; i < kSumRows; ++i) v += s[i][c];
  float* to = at < kD ? dq_weight : dk_weight;
  if (to) to[at & (kD - 1)] = (float)v;
}

// Tokens of a work-group (32, 18 and 5 heads in all, token by token in memory, us of a call in a graph).
// * 1 where there are few tokens, and heads enough for its lanes: 128 tokens 3.4 2.8 3.4, with 4 4.0 3.7 2.8; 512 4.3 3.3 3.7 and 4.4
//   3.9 2.9; 640 4.9 3.7 3.8 and 4.8 3.9 3.0; 1280 9.4 5.9 6.2 and 7.6 5.0 3.3.
// * 4 beyond, 8 where tokens are many and the query heads no more than one load of 4 rows for each of 4 waves: 1280 tokens 8.2 5.3
//   3.8 with 8, 2560 10.0 7.7 3.8 with 4 and 11.2 8.4 4.2 with 8; 8192 30.4 16.5 10.3 and 30.4 14.6 7.6; 32768 95 67 29 and 103 60 20.
int tokens_of(const NormRotaryArgs& a, int max_len) {
  const int64_t tokens = (int64_t)max_len * a.r.nb;
  if (tokens <= 512 && a.r.hq + a.r.hk > 8) return 1;
  return tokens <= 2560 || a.r.hq > 16 ? 4 : 8;
}
// Backwards the work-groups are one round, so that some take a tile more than others: 4 where that leaves the longest of them fewer
// tokens than 8. Us: 128 tokens 8.0 7.1 7.9 with 1, 8.6 7.9 6.7 with 4; 320 9.8 8.8 9.2 and 9.2 8.4 7.1; 1024 17.8 14.6 14.8 and 12.8
// 11.1 8.0, with 8 14.4 11.6 8.1; 2560 19.4 14.9 10.3 with 4 and 20.3 16.1 10.6 with 8, 4096 26.3 18.0 13.0 and 24.8 16.8 11.3 (two tiles
// against one), 8192 46.7 30.8 15.9 and 48.0 31.0 15.9.
int grad_tokens_of(const NormRotaryArgs& a, int max_len) {
  const int64_t tokens = (int64_t)max_len * a.r.nb;
  if (tokens <= 256 && a.r.hq + a.r.hk > 8) return 1;
  auto most = [&](int T) { return ((int64_t)((max_len + T - 1) / T) * a.r.nb + kNormParts - 1) / kNormParts * T; };
  return most(4) < most(8) ? 4 : 8;
}

template <bool kBf16, bool kAdjacent>
hipError_t launch(const NormRotaryArgs& a, int max_len, int kept, int groups, hipStream_t s) {
  const int T = groups ? grad_tokens_of(a, max_len) : tokens_of(a, max_len), ntile = (max_len + T - 1) / T;
  const dim3 block(kThreads);
  if (groups) {
    if (T == 1) hipLaunchKernelGGL((k_norm_rotary_grad<kBf16, kAdjacent, 1>), dim3(groups), block, 0, s, a, ntile, kept);
    else if (T == 4) hipLaunchKernelGGL((k_norm_rotary_grad<kBf16, kAdjacent, 4>), dim3(groups), block, 0, s, a, ntile, kept);
    else hipLaunchKernelGGL((k_norm_rotary_grad<kBf16, kAdjacent, 8>), dim3(groups), block, 0, s, a, ntile, kept);
  } else {
    const dim3 grid((unsigned)std::min<int64_t>((int64_t)ntile * a.r.nb, 1 << 20));
    if (T == 1) hipLaunchKernelGGL((k_norm_rotary<kBf16, kAdjacent, 1>), grid, block, 0, s, a, ntile);
    else if (T == 4) hipLaunchKernelGGL((k_norm_rotary<kBf16, kAdjacent, 4>), grid, block, 0, s, a, ntile);
    else hipLaunchKernelGGL((k_norm_rotary<kBf16, kAdjacent, 8>), grid, block, 0, s, a, ntile);
  }
  return hipGetLastError();
}

hipError_t dispatch(const NormRotaryArgs& a, int dtype, int max_len, int kept, int groups, hipStream_t s) {
  const bool adj = (a.r.flags & OKVQ_ROTARY_ADJACENT) != 0;
  if (dtype == OKVQ_BF16) return adj ? launch<true, true>(a, max_len, kept, groups, s) : launch<true, false>(a, max_len, kept, groups, s);
  return adj ? launch<false, true>(a, max_len, kept, groups, s) : launch<false, false>(a, max_len, kept, groups, s);
}

}  // namespace

hipError_t launch_norm_rotary(const NormRotaryArgs& a, int dtype, int max_len, hipStream_t s) {
  return max_len == 0 ? hipSuccess : dispatch(a, dtype, max_len, 0, 0, s);
}

int norm_rotary_parts(const NormRotaryArgs& a, int max_len) {
  if (max_len == 0) return 0;
  const int T = grad_tokens_of(a, max_len);
  return (int)std::min<int64_t>((int64_t)((max_len + T - 1) / T) * a.r.nb, kNormParts);
}

hipError_t launch_norm_rotary_grad(const NormRotaryArgs& a, int dtype, int max_len, int kept, int groups, hipStream_t s) {
  return groups == 0 ? hipSuccess : dispatch(a, dtype, max_len, kept, groups, s);
}

hipError_t launch_norm_weight_sum(const float* parts, int n, float* dq_weight, float* dk_weight, hipStream_t s) {
  hipLaunchKernelGGL(k_norm_weight_sum, dim3(2 * kD / kSumCols), dim3(kSumCols * kSumRows), 0, s, parts, n, dq_weight, dk_weight);
  return hipGetLastError();
}

}  // namespace okvq
