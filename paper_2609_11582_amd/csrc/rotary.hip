// Rotary positions on several axes, for queries and keys in one launch.
//
// Pair i of a row's 64 channel pairs turns by pos[axis[i]] * inv_freq[i]. The angle is kept as a fraction of a
// turn in 64-bit fixed point: turn[i] = inv_freq[i] / 2 pi in units of 2^-64, and pos * turn[i] modulo 2^64 drops
// whole turns exactly, so position 2^31 is as exact as position 1 (an fp32 angle at position 131072 is off
// by 0.004). The fraction goes through one sincospi in fp32; the rotation is fp32, rounded once.
//
// Bound: memory (one read and one write of every row, 12 bytes of positions a token). A work-group takes
// kTokens tokens: their 64 sines and cosines go to LDS once and serve every head; then 8 lanes carry a row,
// 32 bytes each way, so that whole 256-byte rows move whatever the two layouts are.
#include <algorithm>

#include "q8.hpp"

namespace okvq {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;  // tokens of a work-group

template <bool kBf16, bool kAdjacent>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs p, int ntile) {
  __shared__ __attribute__((aligned(16))) float2 cs[kTokens][64];  // cosine, sine
  const int tid = threadIdx.x, heads = p.hq + p.hk;
  const float dir = (p.flags & OKVQ_ROTARY_INVERSE) ? -1.0f : 1.0f;
  for (int64_t unit = blockIdx.x; unit < (int64_t)ntile * p.nb; unit += gridDim.x) {
    const int bi = (int)(unit / ntile), t0 = (int)(unit % ntile) * kTokens, b = p.b0 + bi;
    const int nt = min(p.lens.lens[bi] - t0, kTokens);
    if (nt <= 0) continue;
    for (int i = tid; i < nt * 64; i += kThreads) {
      const int t = i >> 6, pair = i & 63;
      const int64_t pos = p.pos[((int64_t)b * 3 + p.axis[pair]) * p.n + t0 + t];
      const int32_t frac = (int32_t)(((uint64_t)pos * p.turn[pair]) >> 32);  // turns in units of 2^-32, signed
      float s, c;
      sincospif((float)frac * 0x1p-31f, &s, &c);
      cs[t][pair] = make_float2(c, s * dir);
    }
    __syncthreads();
    for (int i = tid; i < nt * heads * 8; i += kThreads) {
      const int j = i & 7, row = i >> 3, t = row / heads, hh = row - t * heads;
      const bool is_q = hh < p.hq;
      const okvq_rows& in = is_q ? p.q : p.k;
      const okvq_rows& out = is_q ? p.q_out : p.k_out;
      const int h = is_q ? hh : hh - p.hq;
      const uint16_t* src = static_cast<const uint16_t*>(in.data) + (int64_t)b * in.batch_stride + h * in.head_stride +
                            (int64_t)(t0 + t) * in.token_stride;
      uint16_t* dst = static_cast<uint16_t*>(out.data) + (int64_t)b * out.batch_stride + h * out.head_stride +
                      (int64_t)(t0 + t) * out.token_stride;
      // pairs 8 j .. 8 j + 7: neighbouring channels, or the same places of the two halves
      const int at0 = kAdjacent ? 16 * j : 8 * j, at1 = kAdjacent ? 16 * j + 8 : 8 * j + 64;
      const uint4 u = *reinterpret_cast<const uint4*>(src + at0), w = *reinterpret_cast<const uint4*>(src + at1);
      const uint32_t x[8] = {u.x, u.y, u.z, u.w, w.x, w.y, w.z, w.w};
      uint32_t y[8];
      const float4* f = reinterpret_cast<const float4*>(&cs[t][8 * j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 r = f[e];  // cosine and sine of pairs 2 e, 2 e + 1
        if constexpr (kAdjacent) {
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            const float a = row_lo<kBf16>(x[2 * e + d]), c2 = row_hi<kBf16>(x[2 * e + d]);
            const float co = d ? r.z : r.x, si = d ? r.w : r.y;
            y[2 * e + d] = row_pack<kBf16>(__builtin_fmaf(a, co, -(c2 * si)), __builtin_fmaf(c2, co, a * si));
          }
        } else {
          const float a0 = row_lo<kBf16>(x[e]), a1 = row_hi<kBf16>(x[e]);
          const float b0 = row_lo<kBf16>(x[e + 4]), b1 = row_hi<kBf16>(x[e + 4]);
          y[e] = row_pack<kBf16>(__builtin_fmaf(a0, r.x, -(b0 * r.y)), __builtin_fmaf(a1, r.z, -(b1 * r.w)));
          y[e + 4] = row_pack<kBf16>(__builtin_fmaf(b0, r.x, a0 * r.y), __builtin_fmaf(b1, r.z, a1 * r.w));
        }
      }
      *reinterpret_cast<uint4*>(dst + at0) = make_uint4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<uint4*>(dst + at1) = make_uint4(y[4], y[5], y[6], y[7]);
    }
    __syncthreads();  // the next unit overwrites the table
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype, int max_len, hipStream_t s) {
  const int ntile = (max_len + kTokens - 1) / kTokens;
  if (ntile == 0 || a.hq + a.hk == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((int64_t)ntile * a.nb, 1 << 20)), block(kThreads);
  const bool adj = (a.flags & OKVQ_ROTARY_ADJACENT) != 0;
  if (dtype == OKVQ_BF16) {
    if (adj) hipLaunchKernelGGL((k_rotary<true, true>), grid, block, 0, s, a, ntile);
    else hipLaunchKernelGGL((k_rotary<true, false>), grid, block, 0, s, a, ntile);
  } else {
    if (adj) hipLaunchKernelGGL((k_rotary<false, true>), grid, block, 0, s, a, ntile);
    else hipLaunchKernelGGL((k_rotary<false, false>), grid, block, 0, s, a, ntile);
  }
  return hipGetLastError();
}

}  // namespace okvq
