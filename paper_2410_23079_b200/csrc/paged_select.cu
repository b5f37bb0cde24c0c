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
//   a warp, 16 bytes each, and eight pages' loads are under way at once. Scores are left as unsigned keys that sort like the scores.
// pick_kernel: one block per (sequence, KV head) finds the top-th largest key and writes the pages
//   ascending (equal keys: the lowest pages).
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
constexpr int kBatch = 8;            // pages of a lane group whose bounds are under way together

template <typename T, int D>
struct ScorePlan {
  static constexpr int kE = 16 / sizeof(T);
  static constexpr int kChunks = 2 * D / kE;                       // 16-byte chunks of a page's bounds
  static constexpr int kLanes = kChunks < 32 ? kChunks : 32;       // lanes of a page
  static constexpr int kCL = kChunks / kLanes;                     // chunks per lane
  static constexpr int kPages = 32 / kLanes;                       // lane groups of a warp
  static constexpr int kPerBlock = kScoreWarps * kPages * kBatch;
};

template <typename T>
__device__ __forceinline__ void widen(const uint4& u, float (&x)[16 / sizeof(T)]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    else x[i] = __uint_as_float(w[i]);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kScoreWarps * 32) score_kernel(const PagedView w, const SelectArgs a) {
  using L = ScorePlan<T, D>;
  constexpr int kE = L::kE, kLanes = L::kLanes, kCL = L::kCL;
  begin();
  const int b = blockIdx.z, h = blockIdx.y;
  const int len = a.lens[b];
  if (len < 0 || len > a.max_len) return;                   // the pick records it
  const int count = (len + (1 << w.page_log2) - 1) >> w.page_log2;
  if (count <= a.sink + a.recent + a.top) return;
  const int warp = threadIdx.x / 32, wl = threadIdx.x & 31, lane = wl % kLanes, sub = wl / kLanes;
  const int end = count - a.recent;
  const int p0 = a.sink + blockIdx.x * L::kPerBlock + warp * (L::kPages * kBatch) + sub * kBatch;     // this lane group's pages
  if (a.sink + (int)blockIdx.x * L::kPerBlock + warp * (L::kPages * kBatch) >= end) return;           // all of the warp's
  // the pages' bounds, all under way before the first is used
  uint4 raw[kBatch][kCL];
  int mine = -1;                                            // lane i of a group looks up page i
  if (lane < kBatch && p0 + lane < end) {
    mine = a.table[(int64_t)b * a.table_stride + p0 + lane];
    if (mine < 0 || mine >= w.pages) {
      buzz_set_status(w.status, BUZZ_ERR_INVALID, b, mine);
      mine = -1;
    }
  }
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const int page = __shfl_sync(0xffffffffu, mine, i, kLanes);
    const uint4* src = reinterpret_cast<const uint4*>(w.bounds) + ((size_t)max(page, 0) * w.kv_heads + h) * L::kChunks + lane;
#pragma unroll
    for (int c = 0; c < kCL; ++c) raw[i][c] = page >= 0 ? src[c * kLanes] : make_uint4(0, 0, 0, 0);
  }
  double qs[kCL][kE];
#pragma unroll
  for (int c = 0; c < kCL; ++c) {
    const int at = lane + c * kLanes;
    const bool high = at * kE >= D;                         // the second half of the bounds is the largest values
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + ((size_t)b * w.kv_heads + h) * a.group * D) + at % (D / kE);
#pragma unroll
    for (int e = 0; e < kE; ++e) qs[c][e] = 0.0;
    for (int g = 0; g < a.group; ++g) {
      float x[kE];
      widen<T>(q[g * (D / kE)], x);
#pragma unroll
      for (int e = 0; e < kE; ++e) qs[c][e] += (double)(high ? (x[e] < 0.f ? 0.f : x[e]) : (x[e] < 0.f ? x[e] : 0.f));
    }
  }
  double s[kBatch];
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    s[i] = 0.0;
#pragma unroll
    for (int c = 0; c < kCL; ++c) {
      float x[kE];
      widen<T>(raw[i][c], x);
#pragma unroll
      for (int e = 0; e < kE; ++e) s[i] += qs[c][e] * (double)x[e];
    }
  }
  // sums over the lane group, eight pages at once: each step halves the pages a lane holds
  int off = kLanes / 2;
#pragma unroll
  for (int n = kBatch / 2; n >= 1; n >>= 1) {
    const bool up = lane & off;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const double give = up ? s[i] : s[i + n], keep = up ? s[i + n] : s[i];
      s[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
    }
    off >>= 1;
  }
#pragma unroll
  for (; off > 0; off >>= 1) s[0] += __shfl_xor_sync(0xffffffffu, s[0], off);
  constexpr int kRest = kLanes / kBatch;                    // lanes that now hold one page's sum
  const int i = lane / kRest;
  const int page = __shfl_sync(0xffffffffu, mine, i, kLanes);
  if (lane % kRest == 0 && p0 + i < end)
    a.keys[((size_t)b * w.kv_heads + h) * a.max_pages + p0 + i] = page >= 0 ? ordered_key(s[0]) : 0;      // a bad page is below all others
}

// The pick: a block per (sequence, KV head). A histogram of kBins equal bins over the keys' range, then over
// the bin that holds the border, until that bin is taken whole; two or three rounds where the scores spread.
constexpr int kPickThreads = 1024;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kBins = 2 * kPickThreads;
constexpr int kHeld = 8;             // keys a thread keeps in registers; more are read again each round

__global__ void __launch_bounds__(kPickThreads) pick_kernel(const PagedView w, const SelectArgs a) {
  typedef unsigned long long u64;
  __shared__ int hist[kBins];
  __shared__ u64 ends[2][kPickWarps];
  __shared__ int cnt[2][kPickWarps];
  __shared__ int border, border_rest, border_count;
  begin();
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
  // thread t holds a run of consecutive pages, so that ranks in page order follow from one scan
  const u64* keys = a.keys + ((size_t)b * w.kv_heads + h) * a.max_pages + a.sink;
  const int n = count - a.recent - a.sink, per = (n + kPickThreads - 1) / kPickThreads;
  const int lo = min(tid * per, n), mine = min(per, n - lo);
  u64 held[kHeld];
  u64 small = ~0ull, large = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = i < mine ? keys[lo + i] : 0;
  auto each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < mine) f(held[i], i);
    for (int i = kHeld; i < mine; ++i) f(keys[lo + i], i);
  };
  each([&](u64 k, int) { small = min(small, k); large = max(large, k); });
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    small = min(small, __shfl_xor_sync(0xffffffffu, small, off));
    large = max(large, __shfl_xor_sync(0xffffffffu, large, off));
  }
  if (lane == 0) { ends[0][warp] = small; ends[1][warp] = large; }
  hist[tid] = hist[tid + kPickThreads] = 0;
  __syncthreads();
  small = ends[0][lane];
  large = ends[1][lane];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    small = min(small, __shfl_xor_sync(0xffffffffu, small, off));
    large = max(large, __shfl_xor_sync(0xffffffffu, large, off));
  }
  u64 base = small, span = large - small;        // keys base .. base + span hold the border
  int rest = a.top;                              // how many of them are kept
  u64 above;                                     // keys from here on are kept
  for (;;) {
    const int shift = max(0, 64 - __clzll((long long)span) - 11);
    each([&](u64 k, int) { if (k - base <= span) atomicAdd(&hist[(int)((k - base) >> shift)], 1); });
    __syncthreads();
    // bins from the top: thread t has bins kBins - 1 - 2t and the one below it
    const int c0 = hist[kBins - 1 - 2 * tid], c1 = hist[kBins - 2 - 2 * tid];
    int incl = c0 + c1;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += o;
    }
    if (lane == 31) cnt[0][warp] = incl;
    __syncthreads();
    hist[kBins - 1 - 2 * tid] = hist[kBins - 2 - 2 * tid] = 0;
    int over = incl - c0 - c1;
    for (int x = 0; x < kPickWarps; ++x) over += x < warp ? cnt[0][x] : 0;
    if (over < rest && rest <= over + c0 + c1) {
      const bool second = rest > over + c0;
      border = kBins - 1 - 2 * tid - (second ? 1 : 0);
      border_rest = rest - over - (second ? c0 : 0);
      border_count = second ? c1 : c0;
    }
    __syncthreads();
    base += (u64)border << shift;
    rest = border_rest;
    span = (1ull << shift) - 1;
    if (border_count == rest) { above = base; rest = 0; break; }
    if (shift == 0) { above = base + 1; break; }             // equal keys: the first `rest` of them
  }
  // ranks in page order (above wraps to 0 only if base is the largest key there is: then nothing is above)
  const bool none_above = rest > 0 && above == 0;
  int kept = 0, equal = 0;
  each([&](u64 k, int) {
    kept += !none_above && k >= above;
    equal += rest > 0 && k == base;
  });
  int ik = kept, ie = equal;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, ik, off), y = __shfl_up_sync(0xffffffffu, ie, off);
    if (lane >= off) { ik += x; ie += y; }
  }
  if (lane == 31) { cnt[0][warp] = ik; cnt[1][warp] = ie; }
  __syncthreads();
  int at = ik - kept, eq = ie - equal;
  for (int x = 0; x < kPickWarps; ++x) { at += x < warp ? cnt[0][x] : 0; eq += x < warp ? cnt[1][x] : 0; }
  at += min(eq, rest);
  each([&](u64 k, int i) {
    bool take = !none_above && k >= above;
    if (rest > 0 && k == base) take = eq++ < rest;
    if (take) out[a.sink + at++] = a.sink + lo + i;
  });
}

template <typename T, int D>
cudaError_t launch(buzz_paged* c, int layer, const SelectArgs& a, cudaStream_t s) {
  const int middle = a.max_pages - a.sink - a.recent;
  if (a.top > 0 && middle > a.top) {
    const int per = ScorePlan<T, D>::kPerBlock;
    const dim3 grid((middle + per - 1) / per, c->sh.kv_heads, a.batch);
    if (cudaError_t e = buzz_launch_chained(score_kernel<T, D>, grid, kScoreWarps * 32u, 0, s, c->view(layer), a); e != cudaSuccess) return e;
    c->launches += 1;
  }
  const cudaError_t e = buzz_launch_chained(pick_kernel, dim3(c->sh.kv_heads, a.batch), (unsigned)kPickThreads, 0, s, c->view(layer), a);
  if (e == cudaSuccess) c->launches += 1;
  return e;
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
