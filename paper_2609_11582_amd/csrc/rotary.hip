// Rotary positions on several axes, for queries and keys in one launch.
//
// Pair i of a row's 64 channel pairs turns by pos[axis[i]] * inv_freq[i]. The angle is kept as a fraction of a
// turn in 64-bit fixed point: turn[i] = inv_freq[i] / 2 pi in units of 2^-64, and pos * turn[i] modulo 2^64 drops
// whole turns exactly, so position 2^31 is as exact as position 1 (an fp32 angle at position 131072 is off
// by 0.004). The fraction goes through one sincospi in fp32; the rotation is fp32, rounded once.
//
// Bound: memory (one read and one write of every row, 12 bytes of positions a token). A work-group takes T tokens: their
// sines and cosines go to LDS once, and a lane takes the 8 pairs that it turns into registers for all heads. Eight
// lanes carry a row, 32 bytes each way, so that 128-byte pieces of rows move whatever the two layouts are, and a wave has
// the T rows of a head that follow each other in the caches' layout. T is 8, or 1 (the heads then fill the lanes) up to
// some five work-groups for each compute unit, which 8 tokens each would leave idle: 32 heads x 64 tokens 2.7 us against 5.3, 1024
// tokens 4.5 against 6.4, 8 heads x 1280 tokens 3.5 each, 1536 4.2 against 3.6.
#include <algorithm>

#include "q8.hpp"

namespace okvq {
namespace {

constexpr int kThreads = 256;

template <bool kBf16, bool kAdjacent, int T>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs p, int ntile) {
  __shared__ __attribute__((aligned(16))) float2 cs[T][64];  // cosine, sine
  constexpr int kHeads = 8 / T, kStep = kThreads / 64 * kHeads;  // heads of a wave at once, of the work-group
  const int tid = threadIdx.x, lane = tid & 63, heads = p.hq + p.hk;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 7, t = T == 1 ? 0 : lane >> 3, h0 = T == 1 ? wave * kHeads + (lane >> 3) : wave;
  const float dir = (p.flags & OKVQ_ROTARY_INVERSE) ? -1.0f : 1.0f;
  // channels 8 j .. + 7 and 64 + 8 j .. + 7: pairs 8 j .. + 7, or, of neighbours, 4 j .. + 3 and 32 + 4 j .. + 3
  const int at0 = 8 * j, at1 = 8 * j + 64;
  for (int64_t unit = blockIdx.x; unit < (int64_t)ntile * p.nb; unit += gridDim.x) {
    const int bi = (int)(unit / ntile), t0 = (int)(unit % ntile) * T, b = p.b0 + bi;
    const int nt = min(p.lens.lens[bi] - t0, T);
    if (nt <= 0) continue;
    for (int i = tid; i < nt * 64; i += kThreads) {
      const int pair = i & 63;
      const int64_t pos = p.pos[((int64_t)b * 3 + p.axis[pair]) * p.n + t0 + (i >> 6)];
      const int32_t frac = (int32_t)(((uint64_t)pos * p.turn[pair]) >> 32);  // turns in units of 2^-32, signed
      float s, c;
      sincospif((float)frac * 0x1p-31f, &s, &c);
      cs[i >> 6][pair] = make_float2(c, s * dir);
    }
    __syncthreads();
    if (t < nt) {
      float co[8], si[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pair = kAdjacent ? 4 * j + 2 * (e & 1) + 32 * (e >> 1) : 8 * j + 2 * e;
        const float4 r = *reinterpret_cast<const float4*>(&cs[t][pair]);
        co[2 * e] = r.x;
        si[2 * e] = r.y;
        co[2 * e + 1] = r.z;
        si[2 * e + 1] = r.w;
      }
#pragma unroll 4
      for (int h = h0; h < heads; h += kStep) {
        const bool is_q = h < p.hq;
        const okvq_rows& in = is_q ? p.q : p.k;
        const okvq_rows& out = is_q ? p.q_out : p.k_out;
        const int hh = is_q ? h : h - p.hq;
        const uint16_t* src = static_cast<const uint16_t*>(in.data) + (int64_t)b * in.batch_stride + hh * in.head_stride +
                              (int64_t)(t0 + t) * in.token_stride;
        uint16_t* dst = static_cast<uint16_t*>(out.data) + (int64_t)b * out.batch_stride + hh * out.head_stride +
                        (int64_t)(t0 + t) * out.token_stride;
        const uint4 u = *reinterpret_cast<const uint4*>(src + at0), w = *reinterpret_cast<const uint4*>(src + at1);
        const uint32_t x[8] = {u.x, u.y, u.z, u.w, w.x, w.y, w.z, w.w};
        uint32_t y[8];
        if constexpr (kAdjacent) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float a = row_lo<kBf16>(x[e]), c = row_hi<kBf16>(x[e]);
            y[e] = row_pack<kBf16>(__builtin_fmaf(a, co[e], -(c * si[e])), __builtin_fmaf(c, co[e], a * si[e]));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a0 = row_lo<kBf16>(x[e]), a1 = row_hi<kBf16>(x[e]);
            const float b0 = row_lo<kBf16>(x[e + 4]), b1 = row_hi<kBf16>(x[e + 4]);
            y[e] = row_pack<kBf16>(__builtin_fmaf(a0, co[2 * e], -(b0 * si[2 * e])),
                                   __builtin_fmaf(a1, co[2 * e + 1], -(b1 * si[2 * e + 1])));
            y[e + 4] = row_pack<kBf16>(__builtin_fmaf(b0, co[2 * e], a0 * si[2 * e]),
                                       __builtin_fmaf(b1, co[2 * e + 1], a1 * si[2 * e + 1]));
          }
        }
        *reinterpret_cast<uint4*>(dst + at0) = make_uint4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<uint4*>(dst + at1) = make_uint4(y[4], y[5], y[6], y[7]);
      }
    }
    __syncthreads();  // the next unit overwrites the table
  }
}

constexpr int kFewTokens = 1280;

template <bool kBf16, bool kAdjacent>
hipError_t launch(const RotaryArgs& a, int max_len, hipStream_t s) {
  const int T = (int64_t)max_len * a.nb <= kFewTokens ? 1 : 8, ntile = (max_len + T - 1) / T;
  const dim3 grid((unsigned)std::min<int64_t>((int64_t)ntile * a.nb, 1 << 20)), block(kThreads);
  if (T == 1) hipLaunchKernelGGL((k_rotary<kBf16, kAdjacent, 1>), grid, block, 0, s, a, ntile);
  else hipLaunchKernelGGL((k_rotary<kBf16, kAdjacent, 8>), grid, block, 0, s, a, ntile);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype, int max_len, hipStream_t s) {
  if (max_len == 0 || a.hq + a.hk == 0) return hipSuccess;
  const bool adj = (a.flags & OKVQ_ROTARY_ADJACENT) != 0;
  if (dtype == OKVQ_BF16) return adj ? launch<true, true>(a, max_len, s) : launch<true, false>(a, max_len, s);
  return adj ? launch<false, true>(a, max_len, s) : launch<false, false>(a, max_len, s);
}

}  // namespace okvq
