// Which pages a new token attends to: an upper bound on a page's logits from the smallest and largest
// value of each key dimension, and the best pages per (sequence, KV head).
//
//   score(page) = sum_h sum_d max(q_hd lo_d, q_hd hi_d) = sum_d (Q+_d hi_d + Q-_d lo_d),
//   Q+ = sum_h max(q_h, 0), Q- = sum_h min(q_h, 0)
// so the group's queries collapse into one pair of vectors and a page costs 2 d multiply-adds whatever
// the group. What is read is 2 d elements per page, which HBM bounds. Sums are fp64: the pages around
// the border are chosen or left out as a whole, and in fp32 the order of a sum would decide that.
//
// score_kernel: a block takes a run of pages of one (sequence, KV head); a page belongs to some lanes of
//   a warp, 16 bytes each. Scores are left as unsigned keys that sort like the scores.
// pick_kernel: one block per (sequence, KV head); radix selection of the top-th largest key, eight bits
//   a pass, then one ordered pass that writes the pages ascending (equal keys: the lowest pages).
#include "paged_internal.cuh"

namespace {

using namespace buzz_paged_dev;

struct SelectArgs {
  const void* q;
  const int32_t *lens, *table;
  unsigned long long* keys;     // [batch * kv_heads][max_pages]
  int32_t* selected;
  int table_stride, batch, max_len, max_pages, group, sink, recent, top;
};

// fp64 as an unsigned number of the same order; -0 like +0, NaN above all
__device__ __forceinline__ unsigned long long ordered_key(double x) {
  if (x != x) return ~0ull;
  const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
  return (u >> 63) ? ~u : u | 0x8000000000000000ull;
}

constexpr int kScoreWarps = 8;

template <typename T, int D>
__global__ void __launch_bounds__(kScoreWarps * 32) score_kernel(const PagedView w, const SelectArgs a, int pages_per_block) {
  constexpr int kE = 16 / sizeof(T);
  constexpr int kChunks = 2 * D / kE;                       // 16-byte chunks of a page's bounds
  constexpr int kLanes = kChunks < 32 ? kChunks : 32;       // lanes of a page
  constexpr int kCL = kChunks / kLanes;                     // chunks per lane
  constexpr int kPages = 32 / kLanes;                       // pages a warp works on at a time
  const int b = blockIdx.z, h = blockIdx.y;
  const int len = a.lens[b];
  if (len < 0 || len > a.max_len) return;                   // the pick records it
  const int count = (len + (1 << w.page_log2) - 1) >> w.page_log2;
  if (count <= a.sink + a.recent + a.top) return;
  const int end = min(count - a.recent, a.sink + (int)(blockIdx.x + 1) * pages_per_block);
  const int begin = a.sink + blockIdx.x * pages_per_block;
  if (begin >= end) return;
  const int warp = threadIdx.x / 32, wl = threadIdx.x & 31, lane = wl % kLanes, sub = wl / kLanes;
  double qs[kCL][kE];
#pragma unroll
  for (int c = 0; c < kCL; ++c) {
    const int d0 = (lane + c * kLanes) * kE % D;
    const bool high = (lane + c * kLanes) * kE >= D;        // the second half of the bounds is the largest values
#pragma unroll
    for (int e = 0; e < kE; ++e) qs[c][e] = 0.0;
    for (int g = 0; g < a.group; ++g) {
      const T* q = static_cast<const T*>(a.q) + (((size_t)b * w.kv_heads + h) * a.group + g) * D + d0;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const double x = (double)(float)q[e];
        qs[c][e] += high ? (x < 0.0 ? 0.0 : x) : (x < 0.0 ? x : 0.0);
      }
    }
  }
  unsigned long long* keys = a.keys + ((size_t)b * w.kv_heads + h) * a.max_pages;
  for (int p0 = begin + warp * kPages; p0 < end; p0 += kScoreWarps * kPages) {
    const int lp = p0 + sub;
    double s = 0.0;
    if (lp < end) {
      const int page = a.table[(int64_t)b * a.table_stride + lp];
      if (page >= 0 && page < w.pages) {
        const T* bnd = reinterpret_cast<const T*>(w.bounds) + ((size_t)page * w.kv_heads + h) * 2 * D;
#pragma unroll
        for (int c = 0; c < kCL; ++c)
#pragma unroll
          for (int e = 0; e < kE; ++e) s += qs[c][e] * (double)(float)bnd[(lane + c * kLanes) * kE + e];
      } else {
        if (lane == 0) buzz_set_status(w.status, BUZZ_ERR_INVALID, b, page);
        s = -INFINITY;
      }
    }
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 0 && lp < end) keys[lp] = ordered_key(s);
  }
}

constexpr int kPickThreads = 512;

__global__ void __launch_bounds__(kPickThreads) pick_kernel(const PagedView w, const SelectArgs a) {
  __shared__ int hist[256];
  __shared__ int warp_cnt[2][kPickThreads / 32];
  __shared__ int pick_bin, pick_rest;
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
  const int len = a.lens[b];
  if (len < 0 || len > a.max_len) {
    if (tid == 0) buzz_set_status(w.status, BUZZ_ERR_INVALID, b, len);
    return;
  }
  const int count = (len + (1 << w.page_log2) - 1) >> w.page_log2;
  const int most = a.sink + a.recent + a.top;
  int32_t* out = a.selected + ((size_t)b * w.kv_heads + h) * most;
  if (count <= most) {
    for (int i = tid; i < most; i += kPickThreads) out[i] = i < count ? i : -1;
    return;
  }
  for (int i = tid; i < a.sink; i += kPickThreads) out[i] = i;
  for (int i = tid; i < a.recent; i += kPickThreads) out[a.sink + a.top + i] = count - a.recent + i;
  if (a.top == 0) return;
  const unsigned long long* keys = a.keys + ((size_t)b * w.kv_heads + h) * a.max_pages;
  const int first = a.sink, end = count - a.recent;
  // the top-th largest key: its leading bytes one after the other
  unsigned long long prefix = 0, mask = 0;
  int rest = a.top;                              // how many of the keys that share the prefix are kept
  for (int shift = 56; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kPickThreads) hist[i] = 0;
    __syncthreads();
    for (int i = first + tid; i < end; i += kPickThreads) {
      const unsigned long long key = keys[i];
      if ((key & mask) == prefix) atomicAdd(&hist[(int)(key >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int above = 0, bin = 255;
      for (; bin > 0; --bin) {
        if (above + hist[bin] >= rest) break;
        above += hist[bin];
      }
      pick_bin = bin;
      pick_rest = rest - above;
    }
    __syncthreads();
    prefix |= (unsigned long long)pick_bin << shift;
    mask |= 255ull << shift;
    rest = pick_rest;
  }
  // ordered pass: keys above the prefix, and the first `rest` equal to it
  int done = 0, equal = 0;                       // written so far, equal keys met so far
  for (int i0 = first; i0 < end; i0 += kPickThreads) {
    const int i = i0 + tid;
    const unsigned long long key = i < end ? keys[i] : 0;
    const bool is_eq = i < end && key == prefix, is_above = i < end && key > prefix;
    const unsigned beq = __ballot_sync(0xffffffffu, is_eq);
    if (lane == 0) warp_cnt[0][warp] = __popc(beq);
    __syncthreads();
    int eq_before = equal, eq_all = 0;
    for (int x = 0; x < kPickThreads / 32; ++x) {
      if (x < warp) eq_before += warp_cnt[0][x];
      eq_all += warp_cnt[0][x];
    }
    const bool take = is_above || (is_eq && eq_before + __popc(beq & ((1u << lane) - 1)) < rest);
    const unsigned bt = __ballot_sync(0xffffffffu, take);
    if (lane == 0) warp_cnt[1][warp] = __popc(bt);
    __syncthreads();
    int at = done, all = 0;
    for (int x = 0; x < kPickThreads / 32; ++x) {
      if (x < warp) at += warp_cnt[1][x];
      all += warp_cnt[1][x];
    }
    if (take) out[a.sink + at + __popc(bt & ((1u << lane) - 1))] = i;
    done += all;
    equal += eq_all;
  }
}

template <typename T, int D>
cudaError_t launch(buzz_paged* c, int layer, const SelectArgs& a, cudaStream_t s) {
  const int middle = a.max_pages - a.sink - a.recent;
  if (a.top > 0 && middle > a.top) {
    const int per = 64;
    const dim3 grid((middle + per - 1) / per, c->sh.kv_heads, a.batch);
    score_kernel<T, D><<<grid, kScoreWarps * 32, 0, s>>>(c->view(layer), a, per);
    if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
    c->launches += 1;
  }
  pick_kernel<<<dim3(c->sh.kv_heads, a.batch), kPickThreads, 0, s>>>(c->view(layer), a);
  c->launches += 1;
  return cudaGetLastError();
}

}  // namespace

size_t buzz_paged_decode_workspace(const buzz_paged* c);

static size_t select_workspace(const buzz_paged* c, int batch, int max_len) {
  const size_t pages = ((size_t)max_len + c->sh.page_tokens - 1) / c->sh.page_tokens;
  return (size_t)batch * c->sh.kv_heads * pages * sizeof(unsigned long long);
}

extern "C" int buzz_paged_workspace_bytes(buzz_paged_t c, int batch, int max_len, size_t* decode_bytes, size_t* select_bytes) {
  if (!c || !decode_bytes || !select_bytes || batch < 1 || batch > 65535 || max_len < 0) return BUZZ_ERR_INVALID;
  *decode_bytes = buzz_paged_decode_workspace(c);
  *select_bytes = select_workspace(c, batch, max_len);
  return BUZZ_OK;
}

extern "C" int buzz_paged_select(buzz_paged_t c, int layer, const void* q, const int32_t* lens_dev, const int32_t* table_dev,
                                 int table_stride, int batch, int max_len, int sink, int recent, int top, int32_t* selected,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (!c || !c->buf.bounds || layer < 0 || layer >= c->sh.layers || batch < 1 || batch > 65535 || table_stride < 1) return BUZZ_ERR_INVALID;
  if (max_len < 0 || max_len > (int64_t)table_stride * c->sh.page_tokens) return BUZZ_ERR_INVALID;
  if (sink < 0 || recent < 1 || top < 0 || (int64_t)sink + recent + top > 32768) return BUZZ_ERR_INVALID;
  if (!q || !lens_dev || !table_dev || !selected || !workspace) return BUZZ_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(workspace)) & 15u) return BUZZ_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(lens_dev) | reinterpret_cast<uintptr_t>(table_dev) | reinterpret_cast<uintptr_t>(selected)) & 3u)
    return BUZZ_ERR_INVALID;
  if (workspace_bytes < select_workspace(c, batch, max_len)) return BUZZ_ERR_INVALID;
  SelectArgs a;
  a.q = q; a.lens = lens_dev; a.table = table_dev;
  a.keys = static_cast<unsigned long long*>(workspace);
  a.selected = selected;
  a.table_stride = table_stride; a.batch = batch; a.max_len = max_len;
  a.max_pages = (int)(((int64_t)max_len + c->sh.page_tokens - 1) / c->sh.page_tokens);
  a.group = c->group; a.sink = sink; a.recent = recent; a.top = top;
  (void)cudaGetLastError();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (c->sh.dtype == BUZZ_BF16) e = c->sh.head_dim == 128 ? launch<__nv_bfloat16, 128>(c, layer, a, s) : launch<__nv_bfloat16, 64>(c, layer, a, s);
  else e = c->sh.head_dim == 128 ? launch<float, 128>(c, layer, a, s) : launch<float, 64>(c, layer, a, s);
  return e == cudaSuccess ? BUZZ_OK : BUZZ_ERR_CUDA;
}
