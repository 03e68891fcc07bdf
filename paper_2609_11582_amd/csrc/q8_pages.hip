// Page calls of the 8-bit cache: allocation with copy on write, forks, frees, compaction.
//
// The bookkeeping is integers (tables, lengths, holder counts), on the device so that a captured step needs no
// answer from the host; one work-group of 1024 threads plans a call (a thread a slot, block-wide prefix sums over
// the pages), and the bytes move in a second launch that fills the GPU from the plan's list of copies. Counts of
// holders change by integer atomics, whose order does not matter to the result. Bound: the copies by memory, the
// rest by launches and one pass over page_refs.
#include <algorithm>

#include "q8.hpp"

namespace okvq {
namespace {

constexpr int kPlan = 1024;  // threads of a planning work-group
constexpr int kWaves = kPlan / 64;
static_assert(kPlan >= kQ8MaxBatch, "a thread for each slot");
constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = kCopyThreads * 16 * 4;  // a unit of a copy: four 16-byte moves a thread

// exclusive prefix sum over the work-group; *total: the sum. scratch: kWaves + 1 ints; a barrier before its reuse
// is inside
__device__ __forceinline__ int block_prefix(int v, int* scratch, int* total) {
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) scratch[wave] = x;
  __syncthreads();
  if (threadIdx.x == 0) {
    int s = 0;
    for (int w = 0; w < kWaves; ++w) {
      const int t = scratch[w];
      scratch[w] = s;
      s += t;
    }
    scratch[kWaves] = s;
  }
  __syncthreads();
  *total = scratch[kWaves];
  return scratch[wave] + x - v;
}

__device__ __forceinline__ int cap_of(const Q8Pages& c) { return c.max_pages * c.T; }
__device__ __forceinline__ int len_of(const Q8Pages& c, int b) { return min(max(c.lens[b], 0), cap_of(c)); }

// ids of the pages [lo, P) with (refs > 0) == used, the lowest first, at most `most` of them, to list; returns how
// many there are (or `most`, if as many were found)
__device__ int list_pages(const Q8Pages& c, int lo, int hi, bool used, int most, int* list, int* scratch) {
  int found = 0;
  for (int p0 = lo; p0 < hi && found < most; p0 += 4 * kPlan) {
    const int p = p0 + 4 * (int)threadIdx.x;
    int mine = 0;
    bool hit[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hit[i] = p + i < hi && (c.refs[p + i] > 0) == used;
      mine += hit[i];
    }
    int total;
    int at = found + block_prefix(mine, scratch, &total);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (hit[i]) {
        if (at < most) list[at] = p + i;
        ++at;
      }
    found += total;
  }
  return min(found, most);
}

// Copies of the plan, in units of one layer's kCopyBytes of one page's codes; the scales of a page go with its first unit. Of a
// compaction (places) also every table entry becomes its page's new place, ws.list
__global__ __launch_bounds__(kCopyThreads) void k_q8_copy(Q8Pages c, Q8PageWs ws, bool places) {
  const int tid = threadIdx.x;
  if (places)
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + tid; i < (int64_t)c.B * c.max_pages; i += (int64_t)gridDim.x * kCopyThreads) {
      const int id = c.table[i];
      if (id >= 0 && id < c.P) c.table[i] = ws.list[id];
    }
  const int64_t page_bytes = (int64_t)c.H * c.T * kD;  // of one kind
  const int scales = c.H * (c.T / kW);
  const int per = (int)((page_bytes + kCopyBytes - 1) / kCopyBytes);
  const int64_t units = (int64_t)ws.count[0] * c.L * 2 * per;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int part = (int)(u % per);
    int64_t v = u / per;
    const bool values = v & 1;
    v >>= 1;
    const int layer = (int)(v % c.L), pair = (int)(v / c.L);
    const int64_t from = (int64_t)layer * c.P + ws.pairs[2 * pair], to = (int64_t)layer * c.P + ws.pairs[2 * pair + 1];
    uint8_t* codes = values ? c.v_codes : c.k_codes;
    const uint4* src = reinterpret_cast<const uint4*>(codes + from * page_bytes);
    uint4* dst = reinterpret_cast<uint4*>(codes + to * page_bytes);
    const int64_t at = (int64_t)part * (kCopyBytes / 16) + tid, end = page_bytes / 16;
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i * kCopyThreads < end) x[i] = src[at + i * kCopyThreads];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i * kCopyThreads < end) dst[at + i * kCopyThreads] = x[i];
    if (part == 0) {
      float* sc = values ? c.v_scale : c.k_scale;
      for (int i = tid; i < scales; i += kCopyThreads) sc[to * scales + i] = sc[from * scales + i];
    }
  }
}

__global__ __launch_bounds__(kPlan) void k_q8_extend(Q8Pages c, const int32_t* n_new, int32_t* granted, Q8PageWs ws) {
  __shared__ int scratch[kWaves + 1];
  __shared__ int last_of[kPlan], start_of[kPlan + 1], first_of[kPlan];
  __shared__ int bad, copies;
  const int b = threadIdx.x;
  if (b == 0) bad = copies = 0;
  int len = 0, n = 0, have = 0, last = -1, first = 0, need = 0;
  bool over = false;
  if (b < c.B) {
    len = len_of(c, b);
    n = max(n_new[b], 0);
    over = (int64_t)len + n > cap_of(c);
    have = (len + c.T - 1) / c.T;
    if (n > 0 && len % c.T != 0) {
      last = c.table[(int64_t)b * c.max_pages + have - 1];
      if (last < 0 || last >= c.P) last = -1;
    }
  }
  last_of[b] = last;
  __syncthreads();
  if (over) bad = 1;
  bool copied = false;
  if (last >= 0) {
    int others = c.refs[last];  // holders, less the slots before this one that will let go of the page
    if (others > 1)
      for (int j = 0; j < b; ++j) others -= last_of[j] == last;
    copied = others > 1;
  }
  __syncthreads();  // every count is read before one changes
  if (!over && n > 0) need = (len + n + c.T - 1) / c.T - have + copied;
  if (need > c.P) bad = 1;  // with at most 2^20 pages the sum over 1024 slots fits an int otherwise
  need = min(need, c.P);
  first = have - copied;  // first table entry that gets a page
  int total;
  const int start = block_prefix(need, scratch, &total);
  start_of[b] = start;
  first_of[b] = first;
  if (b == 0) start_of[kPlan] = total;
  int got = 0;
  const bool fits = bad == 0 && total <= c.P;
  if (fits) got = list_pages(c, 0, c.P, false, total, ws.list, scratch);
  if (!fits || got < total) {
    if (b < c.B) granted[b] = 0;
    if (b == 0) {
      c.status[0] = 1;
      ws.count[0] = 0;
    }
    return;
  }
  __syncthreads();  // the list is written
  for (int k = b; k < total; k += kPlan) {
    int lo = 0, hi = kPlan;  // slot with start_of[lo] <= k < start_of[lo + 1]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start_of[mid] <= k) lo = mid;
      else hi = mid;
    }
    const int page = ws.list[k];
    c.table[(int64_t)lo * c.max_pages + first_of[lo] + k - start_of[lo]] = page;
    c.refs[page] = 1;
  }
  if (copied) {
    atomicSub(&c.refs[last], 1);
    const int at = atomicAdd(&copies, 1);
    ws.pairs[2 * at] = last;
    ws.pairs[2 * at + 1] = ws.list[start];
  }
  if (b < c.B) {
    if (n > 0) c.lens[b] = len + n;
    granted[b] = n;
  }
  __syncthreads();
  if (b == 0) ws.count[0] = copies;
}

__device__ void let_go(const Q8Pages& c, int b) {
  const int pages = (len_of(c, b) + c.T - 1) / c.T;
  for (int i = threadIdx.x; i < c.max_pages; i += blockDim.x) {
    int32_t& entry = c.table[(int64_t)b * c.max_pages + i];
    const int id = entry;
    if (i < pages && id >= 0 && id < c.P) atomicSub(&c.refs[id], 1);
    entry = -1;
  }
}

// work-groups (pair, 0): tables and counts; (pair, 1 + layer): the raw rows of the open block
__global__ __launch_bounds__(256) void k_q8_fork(Q8Pages c, LenArgs srcs, LenArgs dsts) {
  const int src = srcs.lens[blockIdx.x], dst = dsts.lens[blockIdx.x];
  const int len = len_of(c, src);
  if (blockIdx.y == 0) {
    let_go(c, dst);
    __syncthreads();
    const int pages = (len + c.T - 1) / c.T;
    for (int i = threadIdx.x; i < pages; i += blockDim.x) {
      const int id = c.table[(int64_t)src * c.max_pages + i];
      c.table[(int64_t)dst * c.max_pages + i] = id;
      if (id >= 0 && id < c.P) atomicAdd(&c.refs[id], 1);
    }
    if (threadIdx.x == 0) c.lens[dst] = len;
    return;
  }
  const int64_t layer = blockIdx.y - 1;
  const int rows = len % kW;
  const int64_t from = (layer * c.B + src) * c.H * kW * 16, to = (layer * c.B + dst) * c.H * kW * 16;  // in 16 bytes
  uint4* k = reinterpret_cast<uint4*>(c.k_stage);
  uint4* v = reinterpret_cast<uint4*>(c.v_stage);
  for (int i = threadIdx.x; i < c.H * rows * 16; i += blockDim.x) {
    const int64_t at = (int64_t)(i / (rows * 16)) * kW * 16 + i % (rows * 16);
    k[to + at] = k[from + at];
    v[to + at] = v[from + at];
  }
}

__global__ __launch_bounds__(256) void k_q8_free(Q8Pages c, LenArgs slots) {
  const int b = slots.lens[blockIdx.x];
  let_go(c, b);
  __syncthreads();
  if (threadIdx.x == 0) c.lens[b] = 0;
}

// The plan of a compaction: copies (page in use at or behind n, free page before n), and where each page goes
__global__ __launch_bounds__(kPlan) void k_q8_compact(Q8Pages c, Q8PageWs ws) {
  __shared__ int scratch[kWaves + 1];
  const int tid = threadIdx.x;
  int mine = 0, n;
  for (int p = tid; p < c.P; p += kPlan) mine += c.refs[p] > 0;
  block_prefix(mine, scratch, &n);
  const int moved = list_pages(c, n, c.P, true, c.P, ws.list, scratch);
  __syncthreads();
  list_pages(c, 0, n, false, moved, ws.list2, scratch);  // as many free pages before n
  __syncthreads();
  for (int k = tid; k < moved; k += kPlan) {
    const int from = ws.list[k], to = ws.list2[k];
    ws.pairs[2 * k] = from;
    ws.pairs[2 * k + 1] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
  __syncthreads();
  // the lists have served: list becomes the new place of every page
  for (int p = tid; p < c.P; p += kPlan) ws.list[p] = p;
  __syncthreads();
  for (int k = tid; k < moved; k += kPlan) ws.list[ws.pairs[2 * k]] = ws.pairs[2 * k + 1];
  if (tid == 0) {
    ws.count[0] = moved;
    c.status[1] = n;
  }
}

hipError_t launch_copy(const Q8Pages& c, const Q8PageWs& w, int most, bool places, hipStream_t s) {
  const int64_t page_bytes = (int64_t)c.H * c.T * kD;
  int64_t units = (int64_t)most * c.L * 2 * ((page_bytes + kCopyBytes - 1) / kCopyBytes);
  if (places) units = std::max(units, ((int64_t)c.B * c.max_pages + kCopyThreads - 1) / kCopyThreads);
  hipLaunchKernelGGL(k_q8_copy, dim3((unsigned)std::min<int64_t>(units, 2048)), dim3(kCopyThreads), 0, s, c, w, places);
  return hipGetLastError();
}

}  // namespace

size_t q8_page_workspace_bytes(int B, int P) {
  const size_t pairs = (size_t)std::max(B, P);
  return (4 + 2 * pairs + 2 * (size_t)P) * sizeof(int32_t);
}

Q8PageWs q8_page_ws(void* ws, int B, int P) {
  Q8PageWs w;
  w.count = static_cast<int32_t*>(ws);
  w.pairs = w.count + 4;
  w.list = w.pairs + 2 * (size_t)std::max(B, P);
  w.list2 = w.list + P;
  return w;
}

hipError_t launch_q8_extend(const Q8Pages& c, const int32_t* n_new, int32_t* granted, void* ws, hipStream_t s) {
  const Q8PageWs w = q8_page_ws(ws, c.B, c.P);
  hipLaunchKernelGGL(k_q8_extend, dim3(1), dim3(kPlan), 0, s, c, n_new, granted, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // A launch of 1.5 us (4.2 instead of 2.8 us a call) where no slot copies, which the host cannot know. In the plan's
  // work-group copies are as fast up to some 100 KB only (4 slots x 4 heads x 32 tokens of one layer 9.9 us against 9.5, of 64
  // tokens 12.2 against 9.9, 28 layers 155 against 22): no cache of several layers has so little to copy
  return launch_copy(c, w, c.B, false, s);
}

hipError_t launch_q8_fork(const Q8Pages& c, const LenArgs& src, const LenArgs& dst, int n, hipStream_t s) {
  hipLaunchKernelGGL(k_q8_fork, dim3(n, 1 + c.L), dim3(256), 0, s, c, src, dst);
  return hipGetLastError();
}

hipError_t launch_q8_free(const Q8Pages& c, const LenArgs& slots, int n, hipStream_t s) {
  hipLaunchKernelGGL(k_q8_free, dim3(n), dim3(256), 0, s, c, slots);
  return hipGetLastError();
}

hipError_t launch_q8_compact(const Q8Pages& c, void* ws, hipStream_t s) {
  const Q8PageWs w = q8_page_ws(ws, c.B, c.P);
  hipLaunchKernelGGL(k_q8_compact, dim3(1), dim3(kPlan), 0, s, c, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_copy(c, w, c.P / 2 + 1, true, s);
}

}  // namespace okvq
