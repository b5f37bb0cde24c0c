// Per-head RMS norm of queries and keys and their rotation by position, one pass over both tensors.
//
//   y = x * rsqrt(mean(x^2) + eps) * w;   (a, b) -> (a cos - b sin, b cos + a sin),  angle = pos * inv_freq
//
// Every row (token, head) is read and written once, so the pass is bound by HBM. A row belongs to
// d / 8 lanes of a warp, eight elements each; the mean square is a butterfly over those lanes, and with
// paired halves an element's partner is eight elements of one other lane (rotary_dim / 2 is a multiple
// of eight), fetched by a shuffle. A block first forms the sines and cosines of its tokens, which all
// heads share: the angle in fp64 (a position of a million times a frequency near one leaves fp32 no
// digits after the point), reduced to half turns there, then sinpi and cospi in fp32 (error below 1e-7).
#include "paged_internal.cuh"

namespace {

using namespace buzz_paged_dev;

constexpr int kThreads = 256;
constexpr int kTokens = 4;          // tokens per block at most

struct RopeArgs {
  const void *q, *k, *qw, *kw;
  void *q_out, *k_out;
  const int32_t* pos;
  const float* inv_freq;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  int tokens, q_heads, kv_heads, rotary, tok_per_block;
  float eps;
};

template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const RopeArgs a) {
  constexpr int kLanes = D / 8;               // lanes of a row
  constexpr int kRows = kThreads / kLanes;    // rows a block works on at a time
  __shared__ float2 turn[kTokens][D / 2];     // (cos, sin)
  const int tid = threadIdx.x;
  const int t0 = blockIdx.x * a.tok_per_block;
  const int nt = min(a.tok_per_block, a.tokens - t0);
  const int half = a.rotary / 2;
  for (int i = tid; i < nt * half; i += kThreads) {
    const int t = i / half, f = i - t * half;
    const double x = (double)a.pos[t0 + t] * (double)a.inv_freq[f] * 0.31830988618379067154;   // angle / pi
    float s, c;
    sincospif((float)(x - 2.0 * rint(0.5 * x)), &s, &c);
    turn[t][f] = make_float2(c, s);
  }
  __syncthreads();
  const int lane = tid % kLanes;
  const int heads = a.q_heads + a.kv_heads;
  const int rows = nt * heads;
  float wq[8], wk[8];
  if (a.qw) load8(static_cast<const T*>(a.qw) + lane * 8, wq);
  if (a.kw) load8(static_cast<const T*>(a.kw) + lane * 8, wk);
  // every lane of a warp makes the same number of rounds, so that the shuffles below are whole
  for (int r0 = blockIdx.y * kRows; r0 < rows; r0 += gridDim.y * kRows) {
    const int r = r0 + tid / kLanes;
    const bool on = r < rows;
    const int t = on ? r / heads : 0, h = on ? r - t * heads : 0;
    const bool is_q = h < a.q_heads;
    const int64_t tok = t0 + t;
    float x[8] = {};
    if (on) {
      const T* src = is_q ? static_cast<const T*>(a.q) + tok * a.q_stride + (int64_t)h * D
                          : static_cast<const T*>(a.k) + tok * a.k_stride + (int64_t)(h - a.q_heads) * D;
      load8(src + lane * 8, x);
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
    if (is_q ? a.qw != nullptr : a.kw != nullptr) {
      const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= inv * (is_q ? wq[i] : wk[i]);
    }
    if constexpr (kInterleaved) {
      if (lane * 8 < a.rotary) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 cs = turn[t][lane * 4 + i];
          const float u = x[2 * i], w = x[2 * i + 1];
          x[2 * i] = u * cs.x - w * cs.y;
          x[2 * i + 1] = w * cs.x + u * cs.y;
        }
      }
    } else {
      const int hl = half / 8;                 // lanes of one half
      const bool low = lane < hl, turned = lane < 2 * hl;
      const int mate = low ? lane + hl : turned ? lane - hl : lane;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float other = __shfl_sync(0xffffffffu, x[i], mate, kLanes);
        if (turned) {
          const float2 cs = turn[t][(low ? lane : mate) * 8 + i];
          x[i] = low ? x[i] * cs.x - other * cs.y : x[i] * cs.x + other * cs.y;
        }
      }
    }
    if (on) {
      T* dst = is_q ? static_cast<T*>(a.q_out) + tok * a.q_out_stride + (int64_t)h * D
                    : static_cast<T*>(a.k_out) + tok * a.k_out_stride + (int64_t)(h - a.q_heads) * D;
      store8(dst + lane * 8, x);
    }
  }
}

template <typename T, int D>
cudaError_t launch(const RopeArgs& a, bool interleaved, dim3 grid, cudaStream_t s) {
  if (interleaved) norm_rope_kernel<T, D, true><<<grid, kThreads, 0, s>>>(a);
  else norm_rope_kernel<T, D, false><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

extern "C" int buzz_norm_rope(const buzz_rope_shape* sh, const void* q, const void* k, const int32_t* positions_dev,
                              const float* inv_freq_dev, const void* q_weight, const void* k_weight, void* q_out,
                              void* k_out, int tokens, void* stream) {
  if (!sh || sh->q_heads < 1 || sh->kv_heads < 1 || sh->q_heads > 65536 || sh->kv_heads > 65536) return BUZZ_ERR_INVALID;
  if (sh->head_dim != 64 && sh->head_dim != 128) return BUZZ_ERR_INVALID;
  if (sh->dtype != BUZZ_F32 && sh->dtype != BUZZ_BF16) return BUZZ_ERR_INVALID;
  if (sh->rotary_dim < 16 || sh->rotary_dim > sh->head_dim || sh->rotary_dim % 16) return BUZZ_ERR_INVALID;
  if (!(sh->eps >= 0.f && sh->eps <= 3.4e38f) || sh->reserved != 0 || tokens < 0) return BUZZ_ERR_INVALID;
  const int64_t unit = sh->dtype == BUZZ_BF16 ? 8 : 4;
  const int64_t qrow = (int64_t)sh->q_heads * sh->head_dim, krow = (int64_t)sh->kv_heads * sh->head_dim;
  if (sh->q_stride < qrow || sh->q_out_stride < qrow || sh->k_stride < krow || sh->k_out_stride < krow) return BUZZ_ERR_INVALID;
  if ((sh->q_stride | sh->q_out_stride | sh->k_stride | sh->k_out_stride) % unit) return BUZZ_ERR_INVALID;
  if (tokens == 0) return BUZZ_OK;
  if (!q || !k || !positions_dev || !inv_freq_dev || !q_out || !k_out) return BUZZ_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(q_weight) || !aligned16(k_weight) ||
      (reinterpret_cast<uintptr_t>(positions_dev) | reinterpret_cast<uintptr_t>(inv_freq_dev)) & 3u)
    return BUZZ_ERR_INVALID;
  RopeArgs a{q, k, q_weight, k_weight, q_out, k_out, positions_dev, inv_freq_dev, sh->q_stride, sh->k_stride, sh->q_out_stride,
             sh->k_out_stride, tokens, sh->q_heads, sh->kv_heads, sh->rotary_dim, 1, sh->eps};
  a.tok_per_block = tokens >= kTokens * 592 ? kTokens : 1;
  const dim3 grid((tokens + a.tok_per_block - 1) / a.tok_per_block, 1);
  (void)cudaGetLastError();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool il = sh->interleaved != 0;
  cudaError_t e;
  if (sh->dtype == BUZZ_BF16)
    e = sh->head_dim == 128 ? launch<__nv_bfloat16, 128>(a, il, grid, s) : launch<__nv_bfloat16, 64>(a, il, grid, s);
  else
    e = sh->head_dim == 128 ? launch<float, 128>(a, il, grid, s) : launch<float, 64>(a, il, grid, s);
  return e == cudaSuccess ? BUZZ_OK : BUZZ_ERR_CUDA;
}
