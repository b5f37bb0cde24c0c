// Per-head RMS norm of queries and keys and their rotation by position, one pass over both tensors.
//
//   y = x * rsqrt(mean(x^2) + eps) * w;   (a, b) -> (a cos - b sin, b cos + a sin),  angle = pos * inv_freq
//
// Every row (token, head) is read and written once, so the pass is bound by HBM. A row belongs to
// d / 8 lanes of a warp, eight elements each; the mean square is a butterfly over those lanes, and with
// paired halves an element's partner is eight elements of one other lane (rotary_dim / 2 is a multiple
// of eight), fetched by a shuffle.
//
// A warp takes a run of heads of ONE token, so that a lane's eight sines and cosines stay in registers
// over all of them (read from shared memory per row they cost bank conflicts that took as long as the
// traffic), and keeps the loads of four rounds of rows under way. Few tokens are cut into more runs, for
// the sake of more warps. Angles are formed in fp64 (a position of a million times a
// frequency near one leaves fp32 no digits after the point), reduced to half turns there, then sinpi and
// cospi in fp32 (error below 1e-7); each lane forms some and the warp shares them.
#include "paged_internal.cuh"

namespace {

using namespace buzz_paged_dev;

constexpr int kWarps = 4;
constexpr int kAhead = 4;           // rounds of rows whose loads are under way together

struct RopeArgs {
  const void *q, *k, *qw, *kw;
  void *q_out, *k_out;
  const int32_t* pos;
  const float* inv_freq;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  int tokens, q_heads, kv_heads, rotary, runs, run_heads;
  float eps;
};

template <typename T>
struct Raw { uint4 w[sizeof(T) / 2]; };        // eight elements as they are stored

template <typename T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[4 * i] = __uint_as_float(r.w[i].x); x[4 * i + 1] = __uint_as_float(r.w[i].y);
      x[4 * i + 2] = __uint_as_float(r.w[i].z); x[4 * i + 3] = __uint_as_float(r.w[i].w);
    }
  }
}

template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kWarps * 32) norm_rope_kernel(const RopeArgs a) {
  constexpr int kLanes = D / 8;               // lanes of a row
  constexpr int kRows = 32 / kLanes;          // rows of a warp's round
  __shared__ float2 turn[kWarps][D / 2];      // (cos, sin) of the warp's token
  begin();
  const int warp = threadIdx.x / 32, wl = threadIdx.x & 31, lane = wl % kLanes, sub = wl / kLanes;
  const int64_t unit = (int64_t)blockIdx.x * kWarps + warp;
  const int64_t tok = unit / a.runs;
  if (tok >= a.tokens) return;
  const int h0 = (int)(unit - tok * a.runs) * a.run_heads;
  const int h1 = min(h0 + a.run_heads, a.q_heads + a.kv_heads);
  const T* q = static_cast<const T*>(a.q) + tok * a.q_stride + lane * 8;
  const T* k = static_cast<const T*>(a.k) + tok * a.k_stride + lane * 8;
  Raw<T> raw[kAhead];
  auto fetch = [&](int i, int r) {
    if (r < h1) {
      const uint4* src = reinterpret_cast<const uint4*>(r < a.q_heads ? q + (int64_t)r * D : k + (int64_t)(r - a.q_heads) * D);
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e) raw[i].w[e] = __ldcs(src + e);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
#pragma unroll
    for (int e = 0; e < (int)sizeof(T) / 2; ++e) raw[i].w[e] = make_uint4(0, 0, 0, 0);
    fetch(i, h0 + i * kRows + sub);
  }
  const int half = a.rotary / 2;
  const double pos = (double)a.pos[tok] * 0.31830988618379067154;                    // over pi
  for (int f = wl; f < half; f += 32) {
    const double x = pos * (double)a.inv_freq[f];
    float s, c;
    sincospif((float)(x - 2.0 * rint(0.5 * x)), &s, &c);
    turn[warp][f] = make_float2(c, s);
  }
  __syncwarp();
  // a lane's part of the rotation: element i times co[i] plus its partner times si[i]
  const int hl = half / 8;                     // lanes of one half
  const bool turned = kInterleaved ? lane * 8 < a.rotary : lane < 2 * hl;
  const int mate = !turned ? lane : lane < hl ? lane + hl : lane - hl;
  float co[8], si[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int f = kInterleaved ? lane * 4 + i / 2 : (lane < hl ? lane : mate) * 8 + i;
    const float2 cs = turned ? turn[warp][f] : make_float2(1.f, 0.f);
    co[i] = cs.x;
    si[i] = (kInterleaved ? i % 2 == 0 : lane < hl) ? -cs.y : cs.y;
  }
  float wq[8], wk[8];
  if (a.qw) load8(static_cast<const T*>(a.qw) + lane * 8, wq);
  if (a.kw) load8(static_cast<const T*>(a.kw) + lane * 8, wk);
  T* qo = static_cast<T*>(a.q_out) + tok * a.q_out_stride + lane * 8;
  T* ko = static_cast<T*>(a.k_out) + tok * a.k_out_stride + lane * 8;
  for (int h = h0; h < h1; h += kAhead * kRows) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (h + i * kRows >= h1) break;          // the same for the whole warp
      const int r = h + i * kRows + sub;
      const bool is_q = r < a.q_heads;
      float x[8];
      unpack<T>(raw[i], x);
      fetch(i, r + kAhead * kRows);            // in place of the rows just taken
      if (a.qw || a.kw) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
#pragma unroll
        for (int off = kLanes / 2; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
        const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
        if (is_q ? a.qw != nullptr : a.kw != nullptr) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= inv * (is_q ? wq[e] : wk[e]);
        }
      }
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float other;
        if constexpr (kInterleaved) other = x[e ^ 1];
        else other = __shfl_sync(0xffffffffu, x[e], mate, kLanes);
        y[e] = turned ? x[e] * co[e] + other * si[e] : x[e];
      }
      if (r < h1) store8(is_q ? qo + (int64_t)r * D : ko + (int64_t)(r - a.q_heads) * D, y);
    }
  }
}

template <typename T, int D>
cudaError_t launch(const RopeArgs& a, bool interleaved, unsigned blocks, cudaStream_t s) {
  if (interleaved) return buzz_launch_chained(norm_rope_kernel<T, D, true>, dim3(blocks), kWarps * 32u, 0, s, a);
  return buzz_launch_chained(norm_rope_kernel<T, D, false>, dim3(blocks), kWarps * 32u, 0, s, a);
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
  // A run is a whole token where there are warps enough without cutting one (16 for each of 148 SMs), and at
  // least one round of rows.
  const int heads = sh->q_heads + sh->kv_heads, rows = 32 / (sh->head_dim / 8), rounds = (heads + rows - 1) / rows;
  const int want = (16 * 148 + tokens - 1) / tokens;
  const int per = (rounds + (want < rounds ? want : rounds) - 1) / (want < rounds ? want : rounds);
  RopeArgs a{q, k, q_weight, k_weight, q_out, k_out, positions_dev, inv_freq_dev, sh->q_stride, sh->k_stride, sh->q_out_stride,
             sh->k_out_stride, tokens, sh->q_heads, sh->kv_heads, sh->rotary_dim, (rounds + per - 1) / per, per * rows, sh->eps};
  const int64_t blocks = ((int64_t)tokens * a.runs + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffff) return BUZZ_ERR_TOO_LARGE;
  (void)cudaGetLastError();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool il = sh->interleaved != 0;
  cudaError_t e;
  if (sh->dtype == BUZZ_BF16)
    e = sh->head_dim == 128 ? launch<__nv_bfloat16, 128>(a, il, (unsigned)blocks, s) : launch<__nv_bfloat16, 64>(a, il, (unsigned)blocks, s);
  else
    e = sh->head_dim == 128 ? launch<float, 128>(a, il, (unsigned)blocks, s) : launch<float, 64>(a, il, (unsigned)blocks, s);
  return e == cudaSuccess ? BUZZ_OK : BUZZ_ERR_CUDA;
}
