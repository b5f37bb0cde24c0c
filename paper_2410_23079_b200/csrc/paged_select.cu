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

constexpr int kScoreWarps = 4;
constexpr int kBatch = 8;            // pages of a lane group whose bounds are under way together

template <typename T, int D>
struct ScorePlan {
  static constexpr int kE = 16 / sizeof(T);
  static constexpr int kChunks = 2 * D / kE;                       // 16-byte chunks of a page's bounds
  static constexpr int kLanes = kChunks < 32 ? kChunks : 32;       // lanes of a page
  static constexpr int kCL = kChunks / kLanes;                     // chunks per lane
  static constexpr int kPages = 32 / kLanes;                       // lane groups of a warp
  static constexpr int kBatches = kLanes / kBatch;                 // a lane looks up one page of its group
  static constexpr int kPerBlock = kScoreWarps * 32;
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
  const int tid = threadIdx.x, warp = tid / 32, wl = tid & 31, lane = wl % kLanes, sub = wl / kLanes;
  const int end = count - a.recent, block0 = a.sink + blockIdx.x * L::kPerBlock;
  if (block0 >= end) return;
  // lane i of a group looks up page i of the group's run
  const int p0 = block0 + warp * 32 + sub * kLanes;
  int mine = -1;
  if (p0 + lane < end) {
    mine = a.table[(int64_t)b * a.table_stride + p0 + lane];
    if (mine < 0 || mine >= w.pages) {
      buzz_set_status(w.status, BUZZ_ERR_INVALID, b, mine);
      mine = -1;
    }
  }
  // the group's queries by sign, once per block
  __shared__ double qsum[2 * D];
  for (int i = tid; i < 2 * D; i += kScoreWarps * 32) {
    const T* q = static_cast<const T*>(a.q) + ((size_t)b * w.kv_heads + h) * a.group * D + i % D;
    double sum = 0.0;
    for (int g = 0; g < a.group; ++g) {
      const float x = (float)q[g * D];
      sum += (double)((x < 0.f) == (i < D) || x != x ? x : 0.f);    // the first half of the bounds is the smallest values
    }
    qsum[i] = sum;
  }
  uint4 raw[kBatch][kCL];
  auto fetch = [&](int batch) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int page = __shfl_sync(0xffffffffu, mine, batch * kBatch + i, kLanes);
      const uint4* src = reinterpret_cast<const uint4*>(w.bounds) + ((size_t)max(page, 0) * w.kv_heads + h) * L::kChunks + lane;
#pragma unroll
      for (int c = 0; c < kCL; ++c) raw[i][c] = page >= 0 ? src[c * kLanes] : make_uint4(0, 0, 0, 0);
    }
  };
  fetch(0);
  __syncthreads();
  double qs[kCL][kE];
#pragma unroll
  for (int c = 0; c < kCL; ++c)
#pragma unroll
    for (int e = 0; e < kE; ++e) qs[c][e] = qsum[(lane + c * kLanes) * kE + e];
#pragma unroll 1
  for (int batch = 0; batch < L::kBatches; ++batch) {
    if (block0 + warp * 32 + batch * kBatch >= end) break;    // nothing left for any group of the warp
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
    if (batch + 1 < L::kBatches) fetch(batch + 1);
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
    const int i = batch * kBatch + lane / kRest;
    const int page = __shfl_sync(0xffffffffu, mine, i, kLanes);
    if (lane % kRest == 0 && p0 + i < end)
      a.keys[((size_t)b * w.kv_heads + h) * a.max_pages + p0 + i] = page >= 0 ? ordered_key(s[0]) : 0;      // a bad page is below all others
  }
}

// The pick: a block per (sequence, KV head). A histogram of kBins equal bins over the keys' range finds the
// bin that holds the border; its keys (a handful where the scores spread) are ranked against one another,
// and the one of the wanted rank is the last that is kept. A crowded bin is cut into kBins once more, down
// to single values; pages of one value are ranked by their number.
constexpr int kPickThreads = 1024;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kBins = 2 * kPickThreads;
constexpr int kHeld = 8;             // keys a thread keeps in registers; more are read again each time
constexpr int kRanked = 256;         // keys that are ranked directly

__global__ void __launch_bounds__(kPickThreads) pick_kernel(const PagedView w, const SelectArgs a) {
  typedef unsigned long long u64;
  __shared__ int hist[kBins];
  __shared__ u64 ends[2][kPickWarps];
  __shared__ u64 cand[kRanked];
  __shared__ int cand_at[kRanked];
  __shared__ int cnt[kPickWarps];
  __shared__ int border, border_rest, border_count, cand_n, last_at;
  __shared__ u64 last_key;
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
  // key i of the thread is that of page i * kPickThreads + tid of the middle
  const u64* keys = a.keys + ((size_t)b * w.kv_heads + h) * a.max_pages + a.sink;
  const int n = count - a.recent - a.sink;
  u64 held[kHeld];
  u64 small = ~0ull, large = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = i * kPickThreads + tid < n ? keys[i * kPickThreads + tid] : 0;
  auto each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i * kPickThreads + tid < n) f(held[i], i * kPickThreads + tid);
    for (int i = kHeld * kPickThreads + tid; i < n; i += kPickThreads) f(keys[i], i);
  };
  each([&](u64 k, int) { small = min(small, k); large = max(large, k); });
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    small = min(small, __shfl_xor_sync(0xffffffffu, small, off));
    large = max(large, __shfl_xor_sync(0xffffffffu, large, off));
  }
  if (lane == 0) { ends[0][warp] = small; ends[1][warp] = large; }
  hist[tid] = hist[tid + kPickThreads] = 0;
  if (tid == 0) cand_n = 0;
  __syncthreads();
  small = ends[0][lane];
  large = ends[1][lane];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    small = min(small, __shfl_xor_sync(0xffffffffu, small, off));
    large = max(large, __shfl_xor_sync(0xffffffffu, large, off));
  }
  u64 base = small, span = large - small;        // keys base .. base + span hold the border
  int rest = a.top, shift;                       // how many of them are kept
  for (;;) {
    shift = max(0, 64 - __clzll((long long)span) - 11);
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
    if (lane == 31) cnt[warp] = incl;
    __syncthreads();
    hist[kBins - 1 - 2 * tid] = hist[kBins - 2 - 2 * tid] = 0;
    int over = incl - c0 - c1 + (int)__reduce_add_sync(0xffffffffu, lane < warp ? cnt[lane] : 0);
    if (over < rest && rest <= over + c0 + c1) {
      const bool second = rest > over + c0;
      border = kBins - 1 - 2 * tid - (second ? 1 : 0);
      border_rest = rest - over - (second ? c0 : 0);
      border_count = second ? c1 : c0;
    }
    __syncthreads();
    base += (u64)border << shift;
    span = (1ull << shift) - 1;
    rest = border_rest;
    if (border_count <= kRanked || shift == 0) break;
  }
  // the last key that is kept: the one of rank `rest` in the border's bin
  if (border_count <= kRanked) {
    each([&](u64 k, int i) {
      if (k - base <= span) {
        const int at = atomicAdd(&cand_n, 1);
        cand[at] = k;
        cand_at[at] = i;
      }
    });
    __syncthreads();
    const int c = border_count;
    if (tid < c) {
      int rank = 0;
      for (int x = 0; x < c; ++x) rank += cand[x] > cand[tid] || (cand[x] == cand[tid] && cand_at[x] < cand_at[tid]);
      if (rank == rest - 1) { last_key = cand[tid]; last_at = cand_at[tid]; }
    }
  } else {                                       // one value: the page of that rank among its pages
    int seen = 0;
    for (int i0 = 0; i0 < n; i0 += kPickThreads) {
      const bool eq = i0 + tid < n && keys[i0 + tid] == base;
      const unsigned bal = __ballot_sync(0xffffffffu, eq);
      if (lane == 0) cnt[warp] = __popc(bal);
      __syncthreads();
      const int before = seen + (int)__reduce_add_sync(0xffffffffu, lane < warp ? cnt[lane] : 0) + __popc(bal & ((1u << lane) - 1));
      seen += (int)__reduce_add_sync(0xffffffffu, cnt[lane]);
      if (eq && before == rest - 1) { last_key = base; last_at = i0 + tid; }
      __syncthreads();
    }
  }
  __syncthreads();
  // the kept pages in order: ranks of kHeld rows of pages at a time (hist is free: a count per row and warp)
  const u64 lk = last_key;
  const int la = last_at;
  int done = 0;
  for (int r0 = 0; r0 * kPickThreads < n; r0 += kHeld) {
    unsigned bal[kHeld];
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      const int i = (r0 + r) * kPickThreads + tid;
      u64 k = 0;
      if (i < n) k = r0 == 0 ? held[r] : keys[i];
      bal[r] = __ballot_sync(0xffffffffu, i < n && (k > lk || (k == lk && i <= la)));
      if (lane == 0) hist[r * kPickWarps + warp] = __popc(bal[r]);
    }
    __syncthreads();
    if (warp < kHeld) {                          // warp r: the counts of row r become ranks within it
      const int v = hist[warp * kPickWarps + lane];
      int incl = v;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += o;
      }
      hist[warp * kPickWarps + lane] = incl - v;
      if (lane == 31) cnt[warp] = incl;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      if (bal[r] >> lane & 1) out[a.sink + done + hist[r * kPickWarps + warp] + __popc(bal[r] & ((1u << lane) - 1))] = a.sink + (r0 + r) * kPickThreads + tid;
      done += cnt[r];
    }
    __syncthreads();
  }
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
