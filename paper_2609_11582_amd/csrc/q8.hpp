// Rotary positions and the paged 8-bit cache: argument structs, launchers and the device helpers that their
// kernels share (declarations and contracts: include/okvq.h).
#pragma once

#include "okvq.h"
#include "okvq_device.hpp"
#include "q8_plan.hpp"

namespace okvq {

constexpr int kQ8Block = kW * kD;  // bytes of one block of codes: 32 tokens x 128 channels

// ---- rotary --------------------------------------------------------------------------------------
struct RotaryArgs {
  uint64_t turn[64];  // turns per position in units of 2^-64 turn, modulo one turn
  uint8_t axis[64];
  okvq_rows q, k, q_out, k_out;
  const int32_t* pos;
  LenArgs lens;       // rows of sequences b0 .. b0 + nb - 1
  int b0, nb, hq, hk, n;
  uint32_t flags;
};
hipError_t launch_rotary(const RotaryArgs& a, int dtype, int max_len, hipStream_t s);

// ---- head norms with the rotation ----------------------------------------------------------------
struct NormRotaryArgs {
  RotaryArgs r;             // q_out, k_out: the gradients of q and k in the backward pass
  const float* q_weight;
  const float* k_weight;
  float eps;
  okvq_rows q_grad, k_grad; // backward: gradients of what the forward pass wrote
  float* parts;             // backward: [kNormParts][2][128] sums of work-groups
};
constexpr int kNormParts = 768;   // work-groups of a backward pass at most: three to a compute unit, what the registers of 4 and 8
                                  // tokens allow (fp16 rows by one token fit two, but are 256 work-groups at most)
hipError_t launch_norm_rotary(const NormRotaryArgs& a, int dtype, int max_len, hipStream_t s);
int norm_rotary_parts(const NormRotaryArgs& a, int max_len);  // work-groups of one of the launches of a backward pass
// kept: work-groups whose sums hold those of earlier launches
hipError_t launch_norm_rotary_grad(const NormRotaryArgs& a, int dtype, int max_len, int kept, int groups, hipStream_t s);
hipError_t launch_norm_weight_sum(const float* parts, int n, float* dq_weight, float* dk_weight, hipStream_t s);

// ---- 8-bit cache ---------------------------------------------------------------------------------
// One layer of a cache
struct Q8View {
  uint8_t* k_codes;   // [P][H][T][128]
  uint8_t* v_codes;   // [P][H][T/32][4096]
  float* k_scale;     // [P][H][T/32]
  float* v_scale;
  uint16_t* k_stage;  // [B][H][32][128]
  uint16_t* v_stage;
  const int32_t* table;  // [B][max_pages]
  const int32_t* lens;   // [B]
  int H, Hq, P, max_pages;
  int bshift;         // log2(blocks of a page)
};

struct Q8AppendArgs {
  Q8View c;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* n_new;
  int n_max;
};
hipError_t launch_q8_append(const Q8AppendArgs& a, int format, int dtype, int B, int blocks, hipStream_t s);

struct Q8AttendArgs {
  Q8View c;
  const uint16_t* q;
  const int32_t* n_new;
  uint16_t* out;
  float* ws;
  int n_max, G, ntile, cross;
  float qscale;  // sm_scale log2(e)
  Q8Splits splits;
  // a window or a tree: a row sees the sinks and the newest `window` tokens up to its own place
  int window, sinks;
  // a tree: drafts [B][H][n_max][128], masks [B][n_max][words], and records in front of those of tiles with one split
  const uint16_t* kd;
  const uint16_t* vd;
  const uint32_t* visible;
  int words;
  int64_t single;
};
// What a row sees of the cache (template argument of the attention kernels): the tokens up to its own, or all with `cross`;
// of these the sinks and a window; or what precedes a tree of drafts (all, or sinks and window), whose part a merge adds
constexpr int kQ8Full = 0, kQ8Window = 1, kQ8Tree = 2;
hipError_t launch_q8_prompt(const Q8AttendArgs& a, const Q8Plan& p, int span, int format, int dtype, hipStream_t s);
hipError_t launch_q8_wide(const Q8AttendArgs& a, const Q8Plan& p, int span, int format, int dtype, hipStream_t s);
hipError_t launch_q8_attention(Q8AttendArgs& a, const Q8Plan& p, int span, int format, int dtype, hipStream_t s);
hipError_t launch_q8_tree_merge(const Q8AttendArgs& a, const Q8Plan& p, int dtype, hipStream_t s);

// Page calls, on the whole cache
struct Q8Pages {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float* k_scale;
  float* v_scale;
  uint16_t* k_stage;
  uint16_t* v_stage;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int32_t* status;
  int L, B, H, P, T, max_pages;
};
// Workspace: word 0 the number of copies, then from word 4 their (from, to) pairs, then lists of page ids
struct Q8PageWs {
  int32_t* count;
  int32_t* pairs;  // [max(P, B)][2]
  int32_t* list;   // [P]
  int32_t* list2;  // [P]
};
size_t q8_page_workspace_bytes(int B, int P);
Q8PageWs q8_page_ws(void* ws, int B, int P);
hipError_t launch_q8_extend(const Q8Pages& c, const int32_t* n_new, int32_t* granted, void* ws, hipStream_t s);
hipError_t launch_q8_fork(const Q8Pages& c, const LenArgs& src, const LenArgs& dst, int n, hipStream_t s);
hipError_t launch_q8_free(const Q8Pages& c, const LenArgs& slots, int n, hipStream_t s);
hipError_t launch_q8_compact(const Q8Pages& c, void* ws, hipStream_t s);

// ---- device helpers ------------------------------------------------------------------------------
// two 16-bit values of a dword in fp32; kBf16: bfloat16, else IEEE half
template <bool kBf16>
__device__ __forceinline__ float row_lo(uint32_t w) {
  return kBf16 ? __builtin_bit_cast(float, w << 16) : h2f(w & 0xffffu);
}
template <bool kBf16>
__device__ __forceinline__ float row_hi(uint32_t w) {
  return kBf16 ? __builtin_bit_cast(float, w & 0xffff0000u) : h2f(w >> 16);
}
// two fp32 values rounded to nearest even into a dword
template <bool kBf16>
__device__ __forceinline__ uint32_t row_pack(float lo, float hi) {
  if constexpr (kBf16) {
    typedef float float2v __attribute__((ext_vector_type(2)));
    typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{lo, hi}, bf2v));
  } else {
    return f2h(lo) | (f2h(hi) << 16);
  }
}

// A load from a wave-uniform address through the scalar cache: for what earlier launches wrote and this one only
// reads. As a vector load, the wait for it would wait for every load in flight before it
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}
// Page of a block of a sequence, inside the pool whatever the table holds; the block is wave-uniform
__device__ __forceinline__ int q8_page(const int32_t* row, int block, const Q8View& c) {
  const int id = uniform_load(row + min(block >> c.bshift, c.max_pages - 1));
  return min(max(id, 0), c.P - 1);
}
// Index of (page, head, block within the page) among the blocks of a layer
__device__ __forceinline__ int64_t q8_slot(int page, int h, int block, const Q8View& c) {
  return (((int64_t)page * c.H + h) << c.bshift) + (block & ((1 << c.bshift) - 1));
}
__device__ __forceinline__ int q8_len(const Q8View& c, int b) {
  return min(max(uniform_load(c.lens + b), 0), c.max_pages << (c.bshift + 5));
}

}  // namespace okvq
