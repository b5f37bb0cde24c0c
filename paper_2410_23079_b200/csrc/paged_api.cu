// The paged cache's host object: checks of its shape and buffers, and its status words.
#include <new>

#include "paged_internal.cuh"

namespace {
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

// All rows of a pool as bytes, in swizzled boxes of one tile.
bool make_map(CUtensorMap* map, void* base, size_t rows, int row_bytes, int page_tokens) {
  static EncodeTiledFn encode = nullptr;
  if (!encode) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return false;
    }
    encode = reinterpret_cast<EncodeTiledFn>(p);
  }
  const cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)row_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)buzz_paged_box_bytes(row_bytes), (cuuint32_t)buzz_paged_box_rows(row_bytes, page_tokens)};
  const cuuint32_t steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                box[0] == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
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
  const size_t rows = (size_t)s->layers * s->pages * s->kv_heads * s->page_tokens;
  if ((double)s->layers * s->pages * s->kv_heads * s->page_tokens > 2147483647.0) return BUZZ_ERR_TOO_LARGE;   // a row is a 32-bit coordinate
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
  if (!make_map(&c->k_map, b->k, rows, (int)(s->head_dim * c->csize), s->page_tokens) ||
      !make_map(&c->v_map, b->v, rows, (int)(s->head_dim * c->csize), s->page_tokens)) {
    delete c;
    return BUZZ_ERR_CUDA;
  }
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
