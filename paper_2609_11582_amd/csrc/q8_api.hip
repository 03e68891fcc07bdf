// C ABI of the rotary positions and the paged 8-bit cache: argument checks and launch planning.
// Declarations and contracts: include/okvq.h.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <utility>

#include "q8.hpp"

using namespace okvq;

namespace {

bool aligned16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
okvq_status hip_status(hipError_t e) { return e == hipSuccess ? OKVQ_OK : OKVQ_ERR_HIP; }
// a launch holds fewer than 2^32 threads
bool launchable(int64_t groups, int threads) { return groups * threads <= (int64_t)UINT32_MAX; }

okvq_status check_dims(const okvq_q8_dims* d) {
  if (!d) return OKVQ_ERR_INVALID_ARGUMENT;
  if (d->head_dim != 128) return OKVQ_ERR_UNSUPPORTED;
  if (d->layers < 1 || d->batch < 1 || d->num_kv_heads < 1 || d->num_q_heads < 1 || d->num_pages < 1 || d->max_pages < 1)
    return OKVQ_ERR_INVALID_ARGUMENT;
  if (d->num_q_heads % d->num_kv_heads != 0) return OKVQ_ERR_INVALID_ARGUMENT;
  if (d->page_tokens != 32 && d->page_tokens != 64 && d->page_tokens != 128 && d->page_tokens != 256)
    return OKVQ_ERR_INVALID_ARGUMENT;
  if (d->format != OKVQ_Q8_INT8 && d->format != OKVQ_Q8_E4M3) return OKVQ_ERR_INVALID_ARGUMENT;
  if (d->dtype != OKVQ_F16 && d->dtype != OKVQ_BF16) return OKVQ_ERR_INVALID_ARGUMENT;
  if (d->num_q_heads / d->num_kv_heads > 16 || d->batch > kQ8MaxBatch || d->num_kv_heads > 4096 || d->layers > 4096 ||
      d->num_pages > (1 << 20) || (int64_t)d->max_pages * d->page_tokens > (1 << 27))
    return OKVQ_ERR_UNSUPPORTED;
  return OKVQ_OK;
}

okvq_status check_cache(const okvq_q8_cache* c) {
  if (!c) return OKVQ_ERR_INVALID_ARGUMENT;
  const okvq_status st = check_dims(&c->dims);
  if (st != OKVQ_OK) return st;
  for (const void* p : {(const void*)c->k_codes, (const void*)c->v_codes, (const void*)c->k_scale, (const void*)c->v_scale,
                        (const void*)c->k_stage, (const void*)c->v_stage, (const void*)c->block_table,
                        (const void*)c->seq_lens, (const void*)c->page_refs, (const void*)c->status})
    if (!aligned16(p)) return OKVQ_ERR_INVALID_ARGUMENT;
  return OKVQ_OK;
}

int capacity(const okvq_q8_dims& d) { return d.max_pages * d.page_tokens; }

Q8View view(const okvq_q8_cache* c, int layer) {
  const okvq_q8_dims& d = c->dims;
  const int64_t pool = (int64_t)layer * d.num_pages * d.num_kv_heads * d.page_tokens;  // tokens x heads before the layer
  const int64_t stage = (int64_t)layer * d.batch * d.num_kv_heads * kW * kD;
  Q8View v;
  v.k_codes = c->k_codes + pool * kD;
  v.v_codes = c->v_codes + pool * kD;
  v.k_scale = c->k_scale + pool / kW;
  v.v_scale = c->v_scale + pool / kW;
  v.k_stage = c->k_stage + stage;
  v.v_stage = c->v_stage + stage;
  v.table = c->block_table;
  v.lens = c->seq_lens;
  v.H = d.num_kv_heads;
  v.Hq = d.num_q_heads;
  v.P = d.num_pages;
  v.max_pages = d.max_pages;
  v.bshift = d.page_tokens == 32 ? 0 : d.page_tokens == 64 ? 1 : d.page_tokens == 128 ? 2 : 3;
  return v;
}

Q8Pages pages(const okvq_q8_cache* c) {
  const okvq_q8_dims& d = c->dims;
  return Q8Pages{c->k_codes,     c->v_codes,  c->k_scale,   c->v_scale, c->k_stage, c->v_stage,      c->block_table,
                 c->seq_lens,    c->page_refs, c->status,    d.layers,   d.batch,    d.num_kv_heads,  d.num_pages,
                 d.page_tokens, d.max_pages};
}

// lens_host and n_new_host of a call; n_new may exceed the length where a row may see nothing (empty_rows)
okvq_status check_rows(const okvq_q8_dims& d, const int32_t* lens, const int32_t* n_new, int32_t n_max, bool empty_rows, int* most) {
  *most = 0;
  for (int b = 0; b < d.batch; ++b) {
    if (lens[b] < 0 || n_new[b] < 0 || n_new[b] > n_max) return OKVQ_ERR_INVALID_ARGUMENT;
    if (lens[b] > capacity(d)) return OKVQ_ERR_CAPACITY;
    if (!empty_rows && n_new[b] > lens[b]) return OKVQ_ERR_INVALID_ARGUMENT;
    *most = std::max(*most, n_new[b]);
  }
  return OKVQ_OK;
}

// rows' address of a call with n_max rows: an empty array may be NULL
bool rows_at(const void* p, int32_t n_max) { return aligned16(p) || (p == nullptr && n_max == 0); }

okvq_status check_rows_of(const okvq_rows* r, int32_t n_tokens) {
  if (!rows_at(r->data, n_tokens)) return OKVQ_ERR_INVALID_ARGUMENT;
  for (int64_t s : {r->batch_stride, r->head_stride, r->token_stride})
    if (s < 0 || s % 8 != 0) return OKVQ_ERR_INVALID_ARGUMENT;
  return OKVQ_OK;
}

// Rows that are written may not overlap: by growing stride, a dimension steps over all rows of those before it
bool rows_apart(const okvq_rows& r, int64_t batch, int64_t heads, int64_t tokens) {
  std::pair<int64_t, int64_t> dim[3] = {{r.batch_stride, batch}, {r.head_stride, heads}, {r.token_stride, tokens}};
  std::sort(dim, dim + 3);
  __int128 span = kD;
  for (const auto& [stride, n] : dim) {
    if (n > 1 && stride < span) return false;
    if (n > 1) span += (__int128)stride * (n - 1);
  }
  return true;
}

// f / 2 pi modulo one (positions are whole numbers) in units of 2^-64: f's 53 bits times 2^66 / 2 pi in whole numbers, so that
// it is off by max(|f| / 2 pi, 1) units at most. A double's quotient is 2^-53 off, 2^-22 of f at position 2^31; one in
// extended precision costs the host 5 us for 64 frequencies, this 0.1.
uint64_t turn_fraction(double f) {
  uint64_t bits;
  std::memcpy(&bits, &f, sizeof(bits));
  const int field = (int)(bits >> 52 & 2047);
  const uint64_t m = (bits & ((1ull << 52) - 1)) | (field ? 1ull << 52 : 0);
  const int shift = std::max(field, 1) - 1075 - 2;  // |f| = m 2^(field - 1075)
  const unsigned __int128 p = (unsigned __int128)m * 0xa2f9836e4e44152aull;  // 2^66 / 2 pi
  const uint64_t t = shift <= -128 || shift >= 64 ? 0 : shift <= 0 ? (uint64_t)(p >> -shift) : (uint64_t)p << shift;
  return bits >> 63 ? 0 - t : t;
}

// distinct slots of B; `seen` marks them (arrays on the stack: nothing here throws)
okvq_status check_slots(const int32_t* slots, int n, int B, bool (&seen)[kQ8MaxBatch]) {
  for (int i = 0; i < n; ++i) {
    if (slots[i] < 0 || slots[i] >= B || seen[slots[i]]) return OKVQ_ERR_INVALID_ARGUMENT;
    seen[slots[i]] = true;
  }
  return OKVQ_OK;
}

LenArgs slot_args(const int32_t* slots, int i0, int n) {
  LenArgs a{};
  std::copy(slots + i0, slots + i0 + n, a.lens);
  return a;
}

}  // namespace

extern "C" {

okvq_status okvq_rotary(const okvq_rotary_params* params, int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t n_tokens,
                        const okvq_rows* q, const okvq_rows* k, const int32_t* positions, const int32_t* lens_host,
                        const okvq_rows* q_out, const okvq_rows* k_out, int32_t dtype, uint32_t flags, void* stream) {
  if (!params || batch < 1 || batch > 65535 || n_tokens < 0 || !rows_at(positions, n_tokens)) return OKVQ_ERR_INVALID_ARGUMENT;
  if (flags & ~(uint32_t)(OKVQ_ROTARY_INVERSE | OKVQ_ROTARY_ADJACENT)) return OKVQ_ERR_INVALID_ARGUMENT;
  if (dtype != OKVQ_F16 && dtype != OKVQ_BF16) return OKVQ_ERR_INVALID_ARGUMENT;
  if (!q != !q_out || !k != !k_out || (!q && !k)) return OKVQ_ERR_INVALID_ARGUMENT;
  if ((q && q_heads < 1) || (k && kv_heads < 1)) return OKVQ_ERR_INVALID_ARGUMENT;
  const int hq = q ? q_heads : 0, hk = k ? kv_heads : 0;
  if ((int64_t)hq + hk > 65535) return OKVQ_ERR_UNSUPPORTED;
  for (const okvq_rows* r : {q, k, q_out, k_out})
    if (r && check_rows_of(r, n_tokens) != OKVQ_OK) return OKVQ_ERR_INVALID_ARGUMENT;
  RotaryArgs a;
  a.q = a.k = a.q_out = a.k_out = okvq_rows{};
  for (int i = 0; i < 64; ++i) {
    if (params->axis[i] > 2 || !std::isfinite(params->inv_freq[i])) return OKVQ_ERR_INVALID_ARGUMENT;
    a.axis[i] = params->axis[i];
    a.turn[i] = turn_fraction(params->inv_freq[i]);
  }
  if (q) {
    a.q = *q;
    a.q_out = *q_out;
  }
  if (k) {
    a.k = *k;
    a.k_out = *k_out;
  }
  a.pos = positions;
  a.hq = hq;
  a.hk = hk;
  a.n = n_tokens;
  a.flags = flags;
  int longest = lens_host ? 0 : n_tokens;
  if (lens_host)
    for (int b = 0; b < batch; ++b) {
      if (lens_host[b] < 0 || lens_host[b] > n_tokens) return OKVQ_ERR_INVALID_ARGUMENT;
      longest = std::max(longest, lens_host[b]);
    }
  if (longest > 0 && ((q && !rows_apart(*q_out, batch, hq, longest)) || (k && !rows_apart(*k_out, batch, hk, longest))))
    return OKVQ_ERR_INVALID_ARGUMENT;
  for (int b0 = 0; b0 < batch; b0 += kMaxLenArgs) {
    a.b0 = b0;
    a.nb = std::min(kMaxLenArgs, batch - b0);
    int most = 0;
    for (int i = 0; i < a.nb; ++i) {
      a.lens.lens[i] = lens_host ? lens_host[b0 + i] : n_tokens;
      most = std::max(most, a.lens.lens[i]);
    }
    const okvq_status st = hip_status(launch_rotary(a, dtype, most, static_cast<hipStream_t>(stream)));
    if (st != OKVQ_OK) return st;
  }
  return OKVQ_OK;
}

size_t okvq_q8_buffer_bytes(const okvq_q8_dims* d, int32_t which) {
  if (check_dims(d) != OKVQ_OK) return 0;
  const size_t L = d->layers, B = d->batch, H = d->num_kv_heads, P = d->num_pages, T = d->page_tokens;
  switch (which) {
    case OKVQ_Q8_BUF_K_CODES:
    case OKVQ_Q8_BUF_V_CODES: return L * P * H * T * kD;
    case OKVQ_Q8_BUF_K_SCALE:
    case OKVQ_Q8_BUF_V_SCALE: return L * P * H * (T / kW) * sizeof(float);
    case OKVQ_Q8_BUF_K_STAGE:
    case OKVQ_Q8_BUF_V_STAGE: return L * B * H * kW * kD * 2;
    case OKVQ_Q8_BUF_BLOCK_TABLE: return B * d->max_pages * sizeof(int32_t);
    case OKVQ_Q8_BUF_SEQ_LENS: return B * sizeof(int32_t);
    case OKVQ_Q8_BUF_PAGE_REFS: return P * sizeof(int32_t);
    case OKVQ_Q8_BUF_STATUS: return 4 * sizeof(int32_t);
    default: return 0;
  }
}

okvq_status okvq_q8_append(const okvq_q8_cache* cache, int32_t layer, const int32_t* lens_host, const uint16_t* k_new,
                           const uint16_t* v_new, const int32_t* n_new_host, const int32_t* n_new_dev, int32_t n_max,
                           void* stream) {
  okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  const okvq_q8_dims& d = cache->dims;
  if (layer < 0 || layer >= d.layers || !lens_host || !n_new_host || n_max < 0) return OKVQ_ERR_INVALID_ARGUMENT;
  if (!rows_at(k_new, n_max) || !rows_at(v_new, n_max) || !aligned16(n_new_dev)) return OKVQ_ERR_INVALID_ARGUMENT;
  int most;
  st = check_rows(d, lens_host, n_new_host, n_max, false, &most);
  if (st != OKVQ_OK) return st;
  if (most == 0) return OKVQ_OK;
  // blocks that `most` tokens can touch wherever the sequence ends: the lengths on the device decide which
  const int blocks = (int)(((int64_t)most + kW - 2) / kW + 1);
  if (!launchable((int64_t)blocks * d.num_kv_heads * d.batch, 256)) return OKVQ_ERR_UNSUPPORTED;
  Q8AppendArgs a{view(cache, layer), k_new, v_new, n_new_dev, n_max};
  return hip_status(launch_q8_append(a, d.format, d.dtype, d.batch, blocks, static_cast<hipStream_t>(stream)));
}

size_t okvq_q8_workspace_bytes(const okvq_q8_dims* d, int32_t max_seq_len, int32_t n_max) {
  if (check_dims(d) != OKVQ_OK || max_seq_len < 0 || n_max < 1) return 0;
  return q8_workspace_bound(d->num_q_heads / d->num_kv_heads, n_max);
}

okvq_status okvq_q8_attention(const okvq_q8_cache* cache, int32_t layer, const int32_t* lens_host, const uint16_t* q,
                              const int32_t* n_new_host, const int32_t* n_new_dev, int32_t n_max, float sm_scale,
                              uint16_t* out, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream) {
  okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  const okvq_q8_dims& d = cache->dims;
  const float qscale = sm_scale * 1.4426950408889634f;  // log2(e): the kernels' exponentials have base 2
  if (layer < 0 || layer >= d.layers || !lens_host || !n_new_host || n_max < 0 || !std::isfinite(qscale) ||
      (flags & ~(uint32_t)OKVQ_Q8_CROSS))
    return OKVQ_ERR_INVALID_ARGUMENT;
  if (!rows_at(q, n_max) || !aligned16(n_new_dev) || !rows_at(out, n_max)) return OKVQ_ERR_INVALID_ARGUMENT;
  int most;
  st = check_rows(d, lens_host, n_new_host, n_max, true, &most);
  if (st != OKVQ_OK) return st;
  if (most == 0) return OKVQ_OK;
  const int G = d.num_q_heads / d.num_kv_heads;
  // before the plan, whose products stay inside 64 bits for what can be launched
  if (!launchable(((int64_t)most * G + kQ8PromptCols - 1) / kQ8PromptCols * d.num_kv_heads, 512)) return OKVQ_ERR_UNSUPPORTED;
  Q8Plan plan;
  q8_plan(plan, d.batch, d.num_kv_heads, G, most, lens_host, n_new_host);
  if (!aligned16(workspace) || workspace_bytes < q8_workspace_bound(G, most)) return OKVQ_ERR_WORKSPACE;
  const int64_t units = (int64_t)plan.ntile * d.num_kv_heads;
  if (!launchable(plan.splits.order.most * units * q8_layers(plan), 512) ||
      (plan.splits.order.most > 1 && (!launchable(units * plan.splits.order.split_slots * 32, 256) || units > 65535)))
    return OKVQ_ERR_UNSUPPORTED;
  Q8AttendArgs a;
  a.c = view(cache, layer);
  a.q = q;
  a.n_new = n_new_dev;
  a.out = out;
  a.ws = static_cast<float*>(workspace);
  a.n_max = n_max;
  a.G = G;
  a.cross = (flags & OKVQ_Q8_CROSS) ? 1 : 0;
  a.qscale = qscale;
  return hip_status(launch_q8_attention(a, plan, d.format, d.dtype, static_cast<hipStream_t>(stream)));
}

size_t okvq_q8_page_workspace_bytes(const okvq_q8_dims* d) {
  if (check_dims(d) != OKVQ_OK) return 0;
  return q8_page_workspace_bytes(d->batch, d->num_pages);
}

okvq_status okvq_q8_extend(const okvq_q8_cache* cache, const int32_t* n_new_dev, int32_t* granted, void* workspace,
                           size_t workspace_bytes, void* stream) {
  const okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  if (!aligned16(n_new_dev) || !aligned16(granted)) return OKVQ_ERR_INVALID_ARGUMENT;
  if (!aligned16(workspace) || workspace_bytes < okvq_q8_page_workspace_bytes(&cache->dims)) return OKVQ_ERR_WORKSPACE;
  return hip_status(launch_q8_extend(pages(cache), n_new_dev, granted, workspace, static_cast<hipStream_t>(stream)));
}

okvq_status okvq_q8_fork(const okvq_q8_cache* cache, const int32_t* src_host, const int32_t* dst_host, int32_t n,
                         void* stream) {
  okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  if (n < 0 || (n > 0 && (!src_host || !dst_host))) return OKVQ_ERR_INVALID_ARGUMENT;
  const int B = cache->dims.batch;
  if (n > B) return OKVQ_ERR_INVALID_ARGUMENT;
  bool is_dst[kQ8MaxBatch] = {};
  st = check_slots(dst_host, n, B, is_dst);
  if (st != OKVQ_OK) return st;
  for (int i = 0; i < n; ++i)
    if (src_host[i] < 0 || src_host[i] >= B || is_dst[src_host[i]]) return OKVQ_ERR_INVALID_ARGUMENT;
  for (int i = 0; i < n; i += kMaxLenArgs) {
    const int m = std::min(kMaxLenArgs, n - i);
    st = hip_status(launch_q8_fork(pages(cache), slot_args(src_host, i, m), slot_args(dst_host, i, m), m,
                                   static_cast<hipStream_t>(stream)));
    if (st != OKVQ_OK) return st;
  }
  return OKVQ_OK;
}

okvq_status okvq_q8_free(const okvq_q8_cache* cache, const int32_t* slots_host, int32_t n, void* stream) {
  okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  if (n < 0 || n > cache->dims.batch || (n > 0 && !slots_host)) return OKVQ_ERR_INVALID_ARGUMENT;
  bool seen[kQ8MaxBatch] = {};
  st = check_slots(slots_host, n, cache->dims.batch, seen);
  if (st != OKVQ_OK) return st;
  for (int i = 0; i < n; i += kMaxLenArgs) {
    const int m = std::min(kMaxLenArgs, n - i);
    st = hip_status(launch_q8_free(pages(cache), slot_args(slots_host, i, m), m, static_cast<hipStream_t>(stream)));
    if (st != OKVQ_OK) return st;
  }
  return OKVQ_OK;
}

okvq_status okvq_q8_compact(const okvq_q8_cache* cache, void* workspace, size_t workspace_bytes, void* stream) {
  const okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  if (!aligned16(workspace) || workspace_bytes < okvq_q8_page_workspace_bytes(&cache->dims)) return OKVQ_ERR_WORKSPACE;
  return hip_status(launch_q8_compact(pages(cache), workspace, static_cast<hipStream_t>(stream)));
}

okvq_status okvq_q8_status(const okvq_q8_cache* cache, int32_t* status, void* stream) {
  const okvq_status st = check_cache(cache);
  if (st != OKVQ_OK) return st;
  if (!status) return OKVQ_ERR_INVALID_ARGUMENT;
  hipStream_t s = static_cast<hipStream_t>(stream);
  int32_t words[2] = {0, 0};
  if (hipMemcpyAsync(words, cache->status, sizeof(words), hipMemcpyDeviceToHost, s) != hipSuccess ||
      hipStreamSynchronize(s) != hipSuccess)
    return OKVQ_ERR_HIP;
  status[0] = words[0];
  status[1] = words[1];
  return OKVQ_OK;
}

}  // extern "C"
