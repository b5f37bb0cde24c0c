// The paged cache's host object: checks of its shape and buffers, and its status words.
#include <new>

#include "paged_internal.cuh"

namespace {
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
}  // namespace

extern "C" {

int buzz_paged_create(buzz_paged_t* out, const buzz_paged_shape* s, const buzz_paged_buffers* b) {
  if (!out) return BUZZ_ERR_INVALID;
  *out = nullptr;
  if (!s || !b) return BUZZ_ERR_INVALID;
  if (s->layers < 1 || s->pages < 1 || s->q_heads < 1 || s->kv_heads < 1 || s->q_heads % s->kv_heads) return BUZZ_ERR_INVALID;
  const int g = s->q_heads / s->kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 8) return BUZZ_ERR_INVALID;
  if (s->kv_heads > 65535) return BUZZ_ERR_INVALID;                       // grids hold a KV head per row
  if (s->head_dim != 64 && s->head_dim != 128) return BUZZ_ERR_INVALID;
  if (s->dtype != BUZZ_F32 && s->dtype != BUZZ_BF16) return BUZZ_ERR_INVALID;
  if (s->cache_dtype != s->dtype && s->cache_dtype != BUZZ_E4M3 && s->cache_dtype != BUZZ_I8) return BUZZ_ERR_INVALID;
  if (s->flags & ~BUZZ_FLAG_LOGN) return BUZZ_ERR_INVALID;
  int log2p = 4;
  while (log2p < 7 && (1 << log2p) != s->page_tokens) ++log2p;
  if ((1 << log2p) != s->page_tokens) return BUZZ_ERR_INVALID;
  const bool scaled = s->cache_dtype == BUZZ_E4M3 || s->cache_dtype == BUZZ_I8;
  if (!b->k || !b->v || !b->status || (scaled && (!b->k_scale || !b->v_scale))) return BUZZ_ERR_INVALID;
  if (!aligned16(b->k) || !aligned16(b->v) || !aligned16(b->k_scale) || !aligned16(b->v_scale) || !aligned16(b->bounds) || !aligned16(b->status))
    return BUZZ_ERR_INVALID;
  buzz_paged* c = new (std::nothrow) buzz_paged();
  if (!c) return BUZZ_ERR_INVALID;
  c->sh = *s;
  c->buf = *b;
  if (!scaled) c->buf.k_scale = c->buf.v_scale = nullptr;
  c->group = g;
  c->page_log2 = log2p;
  c->esize = s->dtype == BUZZ_BF16 ? 2 : 4;
  c->csize = scaled ? 1 : c->esize;
  c->launches = 0;
  c->sm_count = 148;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && sms > 0)
    c->sm_count = sms;
  else
    (void)cudaGetLastError();
  if (cudaMemset(b->status, 0, 4 * sizeof(int32_t)) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    delete c;
    return BUZZ_ERR_CUDA;
  }
  *out = c;
  return BUZZ_OK;
}

void buzz_paged_destroy(buzz_paged_t c) { delete c; }

int buzz_paged_status(buzz_paged_t c, void* stream) {
  if (!c) return BUZZ_ERR_INVALID;
  if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return BUZZ_ERR_CUDA;
  int32_t word[4];
  if (cudaMemcpy(word, c->buf.status, sizeof(word), cudaMemcpyDeviceToHost) != cudaSuccess) return BUZZ_ERR_CUDA;
  if (word[0] != 0 && cudaMemset(c->buf.status, 0, sizeof(word)) != cudaSuccess) return BUZZ_ERR_CUDA;
  return word[0];
}

int64_t buzz_paged_launch_count(buzz_paged_t c) { return c ? c->launches : 0; }

}  // extern "C"
