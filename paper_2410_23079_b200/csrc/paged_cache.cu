// Rows into the pages and out of them.
//
// append: a warp owns one (sequence, touched page, KV head) and walks the page's new rows, K and V
// together; a row belongs to d / 8 lanes, eight elements each, so that a row is one 16-byte (bf16) or
// 32-byte (fp32) load per lane. 8-bit caches take the row's largest magnitude by a butterfly over its
// lanes, on the bit patterns (as unsigned numbers a NaN is above every infinity, so it is not lost),
// and divide: the quotients are IEEE divisions because a code is decided at the border between two,
// where a product with the reciprocal comes out on the wrong side. Because the whole page belongs to
// the warp, its bounds need no atomics: the smallest and largest value per dimension are kept in
// registers over the rows and joined with the stored ones only if the page has older rows.
// read: the same walk, the other way. Both are bound by the bytes that they move.
#include "paged_internal.cuh"

namespace {

using namespace buzz_paged_dev;

constexpr int kWarps = 8;

// What one warp works on; false: nothing.
struct Span {
  int page;        // physical
  int slot0, slot1;
  int64_t src;     // packed row index of slot0's token
};
__device__ __forceinline__ bool find_span(const PagedView& w, const int32_t* cu, int total_tokens, int max_new, const int32_t* lens,
                                          const int32_t* table, int table_stride, int b, int j, int lane, Span& s) {
  const int P = 1 << w.page_log2;
  const int c0 = cu ? cu[b] : b, c1 = cu ? cu[b + 1] : b + 1;
  const int n = c1 - c0, len = lens[b];
  if (c0 < 0 || n < 0 || c1 > total_tokens || n > max_new || len < n || len > (int64_t)table_stride * P) {
    if (lane == 0) buzz_set_status(w.status, BUZZ_ERR_INVALID, b, len);
    return false;
  }
  const int start = len - n;
  const int lp = (start >> w.page_log2) + j;
  const int first = lp << w.page_log2;              // at most 2^31 - 1: lp is within the table only if it is below len
  if (n == 0 || (int64_t)lp * P >= len) return false;
  s.slot0 = max(start - first, 0);
  s.slot1 = min(len - first, P);
  s.src = (int64_t)c0 + (first + s.slot0 - start);
  s.page = table[(int64_t)b * table_stride + lp];
  if (s.page < 0 || s.page >= w.pages) {
    if (lane == 0) buzz_set_status(w.status, BUZZ_ERR_INVALID, b, s.page);
    return false;
  }
  return true;
}

// Stores eight elements of one row; `lanes` lanes hold the row.
template <typename C, int kLanes>
__device__ __forceinline__ void put_row(char* cache, float* scales, size_t row, int lane, const float (&x)[8], bool on) {
  if constexpr (C::kScaled) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
    float scale = __fdiv_rn(__uint_as_float(top), C::kTop);
    constexpr float kTiny = 7.888609052210118e-31f;          // 2^-100: a row of zeros has codes of zero
    if (scale < kTiny) scale = kTiny;                         // false for NaN, which stays
    if (!on) return;
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = __fdiv_rn(x[4 * i + e], scale);
      if constexpr (C::kTop == 448.f) {
        const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(y[2], y[3]), __NV_SATFINITE, __NV_E4M3);
        w[i] = a | (b << 16);
      } else {
        w[i] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[i] |= ((uint32_t)min(127, max(-127, __float2int_rn(y[e]))) & 0xffu) << (8 * e);
      }
    }
    reinterpret_cast<uint2*>(cache + row * (kLanes * 8))[lane] = make_uint2(w[0], w[1]);
    if (lane == 0) scales[row] = scale;
  } else {
    if (!on) return;
    if constexpr (C::kSize == 2) store8(reinterpret_cast<__nv_bfloat16*>(cache) + row * (kLanes * 8) + lane * 8, x);
    else store8(reinterpret_cast<float*>(cache) + row * (kLanes * 8) + lane * 8, x);
  }
}

template <typename C, int kLanes>
__device__ __forceinline__ void get_row(const char* cache, const float* scales, size_t row, int lane, float (&x)[8]) {
  if constexpr (C::kScaled) {
    const uint2 w = reinterpret_cast<const uint2*>(cache + row * (kLanes * 8))[lane];
    const float scale = scales[row];
    float a[4], b[4];
    codes_to_float<C>(w.x, a);
    codes_to_float<C>(w.y, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i] * scale; x[4 + i] = b[i] * scale; }
  } else if constexpr (C::kSize == 2) {
    load8(reinterpret_cast<const __nv_bfloat16*>(cache) + row * (kLanes * 8) + lane * 8, x);
  } else {
    load8(reinterpret_cast<const float*>(cache) + row * (kLanes * 8) + lane * 8, x);
  }
}

template <typename T, typename C, int D>
__global__ void __launch_bounds__(kWarps * 32)
append_kernel(const PagedView w, const T* __restrict__ k, const T* __restrict__ v, const int32_t* cu, int total_tokens, int max_new,
              const int32_t* lens, const int32_t* table, int table_stride, int touched) {
  constexpr int kLanes = D / 8, kRows = 32 / kLanes;
  begin();
  const int item = blockIdx.x * kWarps + threadIdx.x / 32;
  const int b = blockIdx.y, j = item / w.kv_heads, h = item - j * w.kv_heads;
  if (j >= touched) return;
  const int wl = threadIdx.x & 31, lane = wl % kLanes, sub = wl / kLanes;
  Span s;
  if (!find_span(w, cu, total_tokens, max_new, lens, table, table_stride, b, j, wl, s)) return;
  const size_t base = ((size_t)s.page * w.kv_heads + h) << w.page_log2;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
  for (int r0 = s.slot0; r0 < s.slot1; r0 += kRows) {
    const int r = r0 + sub;
    const bool on = r < s.slot1;
    float x[8] = {}, y[8] = {};
    if (on) {
      const size_t src = ((size_t)(s.src + (r - s.slot0)) * w.kv_heads + h) * D + lane * 8;
      load8(k + src, x);
      load8(v + src, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) { lo[i] = fminf(lo[i], x[i]); hi[i] = fmaxf(hi[i], x[i]); }
    }
    put_row<C, kLanes>(w.k, w.k_scale, base + r, lane, x, on);
    put_row<C, kLanes>(w.v, w.v_scale, base + r, lane, y, on);
  }
  if (w.bounds == nullptr) return;
  T* bnd = reinterpret_cast<T*>(w.bounds) + ((size_t)s.page * w.kv_heads + h) * 2 * D + lane * 8;
  if (s.slot0 > 0) {                                   // older rows: the stored bounds hold them
    float a[8], c[8];
    load8(bnd, a);
    load8(bnd + D, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo[i] = fminf(lo[i], a[i]); hi[i] = fmaxf(hi[i], c[i]); }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int off = kLanes; off < 32; off <<= 1) {
      lo[i] = fminf(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], off));
      hi[i] = fmaxf(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], off));
    }
  }
  if (sub == 0) {
    store8(bnd, lo);
    store8(bnd + D, hi);
  }
}

template <typename T, typename C, int D>
__global__ void __launch_bounds__(kWarps * 32)
read_kernel(const PagedView w, T* __restrict__ k, T* __restrict__ v, const int32_t* cu, int total_tokens, int max_new,
            const int32_t* lens, const int32_t* table, int table_stride, int touched) {
  constexpr int kLanes = D / 8, kRows = 32 / kLanes;
  begin();
  const int item = blockIdx.x * kWarps + threadIdx.x / 32;
  const int b = blockIdx.y, j = item / w.kv_heads, h = item - j * w.kv_heads;
  if (j >= touched) return;
  const int wl = threadIdx.x & 31, lane = wl % kLanes, sub = wl / kLanes;
  Span s;
  if (!find_span(w, cu, total_tokens, max_new, lens, table, table_stride, b, j, wl, s)) return;
  const size_t base = ((size_t)s.page * w.kv_heads + h) << w.page_log2;
  for (int r = s.slot0 + sub; r < s.slot1; r += kRows) {
    float x[8], y[8];
    get_row<C, kLanes>(w.k, w.k_scale, base + r, lane, x);
    get_row<C, kLanes>(w.v, w.v_scale, base + r, lane, y);
    const size_t dst = ((size_t)(s.src + (r - s.slot0)) * w.kv_heads + h) * D + lane * 8;
    store8(k + dst, x);
    store8(v + dst, y);
  }
}

struct Call {
  void *k, *v;
  const int32_t *cu, *lens, *table;
  int batch, total_tokens, max_new, table_stride;
  bool write;
};

template <typename T, typename C, int D>
cudaError_t launch(buzz_paged* c, int layer, const Call& a, cudaStream_t s) {
  const int P = c->sh.page_tokens;
  const int touched = (a.max_new - 1) / P + 2;         // pages that max_new tokens can touch, the first part-filled
  const long long items = (long long)(a.max_new == 1 ? 1 : touched) * c->sh.kv_heads;
  const dim3 grid((unsigned)((items + kWarps - 1) / kWarps), a.batch);
  const int most = a.max_new == 1 ? 1 : touched;
  if (a.write)
    return buzz_launch_chained(append_kernel<T, C, D>, grid, kWarps * 32, 0, s, c->view(layer), (const T*)a.k, (const T*)a.v, a.cu,
                               a.total_tokens, a.max_new, a.lens, a.table, a.table_stride, most);
  return buzz_launch_chained(read_kernel<T, C, D>, grid, kWarps * 32, 0, s, c->view(layer), (T*)a.k, (T*)a.v, a.cu, a.total_tokens,
                             a.max_new, a.lens, a.table, a.table_stride, most);
}

template <typename T, typename C>
cudaError_t launch_d(buzz_paged* c, int layer, const Call& a, cudaStream_t s) {
  return c->sh.head_dim == 128 ? launch<T, C, 128>(c, layer, a, s) : launch<T, C, 64>(c, layer, a, s);
}

int move_rows(buzz_paged* c, int layer, const Call& a, void* stream) {
  if (!c || layer < 0 || layer >= c->sh.layers || a.batch < 1 || a.batch > 65535) return BUZZ_ERR_INVALID;
  if (a.total_tokens < 1 || a.max_new < 1 || a.max_new > a.total_tokens || a.table_stride < 1) return BUZZ_ERR_INVALID;
  if (!a.k || !a.v || !a.lens || !a.table || (!a.cu && a.total_tokens != a.batch)) return BUZZ_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15u) return BUZZ_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(a.cu) | reinterpret_cast<uintptr_t>(a.lens) | reinterpret_cast<uintptr_t>(a.table)) & 3u) return BUZZ_ERR_INVALID;
  (void)cudaGetLastError();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaErrorInvalidValue;
  const bool wide = c->sh.dtype == BUZZ_F32;
  switch (c->sh.cache_dtype) {
    case BUZZ_F32: e = launch_d<float, CacheF32>(c, layer, a, s); break;
    case BUZZ_BF16: e = launch_d<__nv_bfloat16, CacheBF16>(c, layer, a, s); break;
    case BUZZ_E4M3: e = wide ? launch_d<float, CacheE4M3>(c, layer, a, s) : launch_d<__nv_bfloat16, CacheE4M3>(c, layer, a, s); break;
    case BUZZ_I8: e = wide ? launch_d<float, CacheI8>(c, layer, a, s) : launch_d<__nv_bfloat16, CacheI8>(c, layer, a, s); break;
  }
  c->launches += 1;
  return e == cudaSuccess ? BUZZ_OK : BUZZ_ERR_CUDA;
}

}  // namespace

extern "C" int buzz_paged_append(buzz_paged_t c, int layer, const void* k, const void* v, const int32_t* cu_seqlens_dev, int batch,
                                 int total_tokens, int max_new, const int32_t* lens_dev, const int32_t* table_dev, int table_stride,
                                 void* stream) {
  return move_rows(c, layer, Call{const_cast<void*>(k), const_cast<void*>(v), cu_seqlens_dev, lens_dev, table_dev, batch, total_tokens,
                                  max_new, table_stride, true}, stream);
}

extern "C" int buzz_paged_read(buzz_paged_t c, int layer, void* k_out, void* v_out, const int32_t* cu_seqlens_dev, int batch,
                               int total_tokens, int max_new, const int32_t* lens_dev, const int32_t* table_dev, int table_stride,
                               void* stream) {
  return move_rows(c, layer, Call{k_out, v_out, cu_seqlens_dev, lens_dev, table_dev, batch, total_tokens, max_new, table_stride, false}, stream);
}
