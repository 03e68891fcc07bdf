// Codec of the paged 8-bit cache: new tokens of one layer into their pages.
//
// A work-group quantizes one block (32 tokens x 128 channels) of one KV head, keys and values: amax over the
// block's tokens, scale = fl(amax * fl(1 / M)), codes = round(fl(x / scale)). The block that was open before the
// call takes its older rows from the stage, so that chunks do not change the bytes. The division of the rows is
// IEEE, as the contract says: the codes are those of the documented fp32 order.
//
// Bound: memory (512 bytes read, 256 written a token and head). Thread (tgrp, cgrp) holds tokens 4 tgrp ..
// + 3 of channels 4 cgrp .. + 3 of both kinds: 8-byte loads, 32 lanes to a 256-byte row. A key store is then 4
// bytes a row, a value dword is one channel's 4 tokens; the values pass through LDS to leave in whole 16-byte
// slots of the operand order.
#include <type_traits>

#include "q8.hpp"
#include "wave_ops.hpp"

namespace okvq {
namespace {

constexpr int kThreads = 256;

// fl(x / scale) for many x of one scale: the quotient by the scale's correctly rounded reciprocal y, corrected twice by
// its remainder (Markstein's theorem: the first step leaves a faithful quotient, the second the correctly rounded
// one), 5 instructions instead of the 11 of a division (32768 tokens, 4 heads: 29.6 -> 24.5 us with the maxima by DPP). Exact where no remainder
// underflows: at scales below 2^-80, where a remainder that counts could, and above 2^80 the division itself is taken.
struct Ratio {
  float scale, y;
  bool direct;
};
__device__ __forceinline__ Ratio ratio_of(float scale) {
  return Ratio{scale, div_rn(1.0f, scale), !(scale >= 0x1p-80f && scale <= 0x1p80f)};
}
// t = fl(x / scale), clamped
template <int kFmt, bool kDirect>
__device__ __forceinline__ float q8_ratio(float x, const Ratio& r) {
  constexpr float top = kFmt == OKVQ_Q8_INT8 ? 127.0f : 448.0f;
  float t;
  if constexpr (kDirect) {
    t = div_rn(x, r.scale);
  } else {
    const float q0 = x * r.y, q1 = __builtin_fmaf(__builtin_fmaf(-r.scale, q0, x), r.y, q0);
    t = __builtin_fmaf(__builtin_fmaf(-r.scale, q1, x), r.y, q1);
    if constexpr (kFmt == OKVQ_Q8_E4M3) t = __builtin_copysignf(t, x);  // -0 has a code, and its remainder is +0
  }
  return fminf(fmaxf(t, -top), top);
}
// codes of four ratios as the bytes of a dword
template <int kFmt>
__device__ __forceinline__ uint32_t q8_pack(float a, float b, float c, float d) {
  if constexpr (kFmt == OKVQ_Q8_INT8) {
    const uint32_t ab = ((uint32_t)(int)rintf(a) & 0xffu) | (((uint32_t)(int)rintf(b) & 0xffu) << 8);
    return ab | (((uint32_t)(int)rintf(c) & 0xffu) << 16) | ((uint32_t)(int)rintf(d) << 24);
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);  // e4m3, round to nearest even
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
}

template <int kFmt, bool kBf16>
__global__ __launch_bounds__(kThreads) void k_q8_append(Q8AppendArgs p) {
  __shared__ __attribute__((aligned(16))) uint32_t vt[kQ8Block / 4];
  __shared__ float amax_k[4], amax_v[4];
  constexpr float top = kFmt == OKVQ_Q8_INT8 ? 127.0f : 448.0f;
  const Q8View& c = p.c;
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, wave = tid >> 6;
  const int len = q8_len(c, b), n = min(min(max(p.n_new[b], 0), p.n_max), len), old = len - n;
  const int first = old / kW, block = first + (int)blockIdx.x, t0 = block * kW;
  if (n == 0 || t0 >= len) return;
  const int64_t slot = q8_slot(q8_page(c.table + (int64_t)b * c.max_pages, block, c), h, block, c);
  const int cg = tid & 31, tg = tid >> 5;
  const int64_t head = (int64_t)b * c.H + h;
  const uint2* kn = reinterpret_cast<const uint2*>(p.k) + head * p.n_max * 32 + cg;
  const uint2* vn = reinterpret_cast<const uint2*>(p.v) + head * p.n_max * 32 + cg;
  const uint2* ks = reinterpret_cast<const uint2*>(c.k_stage) + head * kW * 32 + cg;
  const uint2* vs = reinterpret_cast<const uint2*>(c.v_stage) + head * kW * 32 + cg;
  // every row from where it is, without a branch; rows behind the last token from its address, and zeroed
  uint2 kr[4], vr[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * tg + i, t = t0 + row;
    const int64_t at = (int64_t)min(t - old, n - 1) * 32;
    kr[i] = *(t < old ? ks + row * 32 : kn + at);
    vr[i] = *(t < old ? vs + row * 32 : vn + at);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t0 + 4 * tg + i >= len) kr[i] = vr[i] = make_uint2(0u, 0u);
  float ka = 0.0f, va = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ka = fmaxf(ka, fmaxf(fmaxf(fabsf(row_lo<kBf16>(kr[i].x)), fabsf(row_hi<kBf16>(kr[i].x))),
                         fmaxf(fabsf(row_lo<kBf16>(kr[i].y)), fabsf(row_hi<kBf16>(kr[i].y)))));
    va = fmaxf(va, fmaxf(fmaxf(fabsf(row_lo<kBf16>(vr[i].x)), fabsf(row_hi<kBf16>(vr[i].x))),
                         fmaxf(fabsf(row_lo<kBf16>(vr[i].y)), fabsf(row_hi<kBf16>(vr[i].y)))));
  }
  ka = wave_max(ka);
  va = wave_max(va);
  if ((tid & 63) == 0) {
    amax_k[wave] = ka;
    amax_v[wave] = va;
  }
  __syncthreads();
  ka = fmaxf(fmaxf(amax_k[0], amax_k[1]), fmaxf(amax_k[2], amax_k[3]));
  va = fmaxf(fmaxf(amax_v[0], amax_v[1]), fmaxf(amax_v[2], amax_v[3]));
  float sk = ka * (1.0f / top), sv = va * (1.0f / top);
  sk = sk > 0.0f ? sk : 1.0f;
  sv = sv > 0.0f ? sv : 1.0f;

  // The open block's raw rows, by the work-group that has read the stage (its loads are complete: the maxima
  // above needed them): the rows of the sequence's last block that came with this call. In the block it read
  // they lie behind the rows it read
  if (blockIdx.x == 0 && (len & (kW - 1)) != 0) {
    const int s0 = max(len / kW * kW, old);
    uint4* kd = reinterpret_cast<uint4*>(c.k_stage) + head * kW * 16;
    uint4* vd = reinterpret_cast<uint4*>(c.v_stage) + head * kW * 16;
    const uint4* k4 = reinterpret_cast<const uint4*>(p.k) + head * p.n_max * 16;
    const uint4* v4 = reinterpret_cast<const uint4*>(p.v) + head * p.n_max * 16;
    for (int i = tid; i < (len - s0) * 16; i += kThreads) {
      const int t = s0 + (i >> 4), ch = i & 15;
      kd[(t & (kW - 1)) * 16 + ch] = k4[(int64_t)(t - old) * 16 + ch];
      vd[(t & (kW - 1)) * 16 + ch] = v4[(int64_t)(t - old) * 16 + ch];
    }
  }

  uint32_t* kd = reinterpret_cast<uint32_t*>(c.k_codes + slot * kQ8Block) + cg;
  // Slot 64 j + 16 g + n of the block is kept at n ^ j within its row of 16: lanes that differ in j alone
  // would otherwise meet in one bank
  const int j = cg >> 3, bb = (cg >> 2) & 1, n0 = (cg & 3) * 4, a = tg >> 2, g = tg & 3;
  const Ratio rk = ratio_of(sk), rv = ratio_of(sv);
  auto code = [&](auto direct) {
    constexpr bool kDirect = decltype(direct)::value;
    float vq[4][4];  // [channel][token]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kd[(4 * tg + i) * 32] =
          q8_pack<kFmt>(q8_ratio<kFmt, kDirect>(row_lo<kBf16>(kr[i].x), rk), q8_ratio<kFmt, kDirect>(row_hi<kBf16>(kr[i].x), rk),
                        q8_ratio<kFmt, kDirect>(row_lo<kBf16>(kr[i].y), rk), q8_ratio<kFmt, kDirect>(row_hi<kBf16>(kr[i].y), rk));
      vq[0][i] = q8_ratio<kFmt, kDirect>(row_lo<kBf16>(vr[i].x), rv);
      vq[1][i] = q8_ratio<kFmt, kDirect>(row_hi<kBf16>(vr[i].x), rv);
      vq[2][i] = q8_ratio<kFmt, kDirect>(row_lo<kBf16>(vr[i].y), rv);
      vq[3][i] = q8_ratio<kFmt, kDirect>(row_hi<kBf16>(vr[i].y), rv);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      vt[((64 * j + 16 * g + ((n0 + e) ^ j)) << 2) + 2 * bb + a] = q8_pack<kFmt>(vq[e][0], vq[e][1], vq[e][2], vq[e][3]);
  };
  if (kBf16 && (rk.direct || rv.direct)) code(std::true_type{});  // fp16 rows have scales of 2^-33 to 2^9
  else code(std::false_type{});
  __syncthreads();
  reinterpret_cast<uint4*>(c.v_codes + slot * kQ8Block)[tid] =
      reinterpret_cast<const uint4*>(vt)[(tid & ~15) | ((tid & 15) ^ (tid >> 6))];
  if (tid == 0) {
    c.k_scale[slot] = sk;
    c.v_scale[slot] = sv;
  }
}

}  // namespace

hipError_t launch_q8_append(const Q8AppendArgs& a, int format, int dtype, int B, int blocks, hipStream_t s) {
  const dim3 grid(blocks, a.c.H, B), block(kThreads);
  if (format == OKVQ_Q8_INT8) {
    if (dtype == OKVQ_BF16) hipLaunchKernelGGL((k_q8_append<OKVQ_Q8_INT8, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_q8_append<OKVQ_Q8_INT8, false>), grid, block, 0, s, a);
  } else {
    if (dtype == OKVQ_BF16) hipLaunchKernelGGL((k_q8_append<OKVQ_Q8_E4M3, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_q8_append<OKVQ_Q8_E4M3, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace okvq
