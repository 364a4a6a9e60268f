// extern "C" entry points of libjfkv.so: host-side validation, TMA tensor-map
// construction and kernel dispatch.  See include/jfkv.h for the contract.
#include <cstdio>
#include <cstring>
#include <mutex>

#include "common.cuh"
#include "latent.cuh"
#include "prefill.cuh"
#include "tq4.cuh"

namespace jfkv {
int launch_append(const Geom&, const jf_kv_pool&, const int32_t*, int32_t, int32_t,
                  const int32_t*, const int32_t*, const void*, const void*, int32_t, int32_t*,
                  cudaStream_t);
int launch_page_copy(const Geom&, const jf_kv_pool&, const int32_t*, int32_t, void*, int32_t*,
                     bool, cudaStream_t);
int launch_decode(const Geom&, const jf_kv_pool&, const CUtensorMap&, const int32_t*, int32_t,
                  const int32_t*, int32_t, const void*, int32_t, float, void*, void*, int32_t,
                  cudaStream_t, const void* k_new = nullptr, const void* v_new = nullptr,
                  int32_t q_len = 1);
size_t decode_workspace_bytes(int64_t B, int64_t Hq, int64_t D, int64_t S);
int tq4_codebook_host(int d, float* out);
int tq4_make_params(const jf_tq4_codec* codec, int d, Tq4Params* p);
int launch_tq4_append(const Geom&, const jf_kv_pool&, const Tq4Params&, const int32_t*, int32_t,
                      int32_t, const int32_t*, const int32_t*, const void*, const void*, int32_t,
                      int32_t*, cudaStream_t);
int launch_tq4_decode(const Geom&, const jf_kv_pool&, const CUtensorMap&, const Tq4Params&,
                      const int32_t*, int32_t, const int32_t*, int32_t, const void*, int32_t,
                      float, void*, void*, int32_t, cudaStream_t, const void*, const void*,
                      int32_t);
int decode_box_rows();
int launch_prefill(const Geom&, const jf_kv_pool&, const CUtensorMap&, const int32_t*,
                   const void*, int32_t, int32_t, int32_t, float, int32_t, void*, void*,
                   cudaStream_t);
int launch_prefill_batch(const Geom&, const jf_kv_pool&, const int32_t* const*, const int32_t*,
                         const int32_t*, const void*, const int64_t*, int32_t, int32_t, float,
                         int32_t, void*, void*, cudaStream_t, int32_t, int64_t,
                         const Tq4Params*, const P8Plan* plan = nullptr);
size_t prefill_workspace_bytes(int64_t rows, int64_t Hq, int64_t D, int64_t S, int fmt);
int launch_rope(const jf_rope&, const int32_t*, int64_t, int32_t, int32_t, const jf_rope_rows&,
                const jf_rope_rows&, int32_t, int32_t, cudaStream_t);
int launch_kv8_rows(const Geom&, const jf_kv_pool&, const int32_t*, int32_t, int32_t,
                    const int32_t*, const int32_t*, void*, int64_t, void*, int64_t, int32_t,
                    int32_t*, bool, cudaStream_t);
int kv8_box_rows();
int64_t kv8_score_floats(int64_t G, int64_t wstride);
int launch_kv8_decode(const Geom&, const jf_kv_pool&, const CUtensorMap&, const int32_t*, int32_t,
                      const int32_t*, int32_t, const void*, int32_t, float, void*, void*, int32_t,
                      float*, const float*, float*, int64_t, cudaStream_t);
int launch_kv8_evict(const Geom&, const jf_kv_pool&, const int32_t*, int32_t, const int32_t*,
                     int32_t, const float*, int64_t, int32_t, int32_t, int32_t, const int32_t*,
                     int32_t, int32_t*, float*, int32_t*, int32_t*, cudaStream_t);
int sm_count();
}  // namespace jfkv

using namespace jfkv;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_pool(const jf_kv_pool* pool) {
  if (!pool || !pool->base) return JF_ERR_INVALID_ARG;
  if (!aligned(pool->base, 16)) return JF_ERR_INVALID_ARG;
  if (pool->num_pages < 1 || pool->num_kv_heads < 1) return JF_ERR_INVALID_ARG;
  if (pool->format != JF_FMT_AFFINE4_G64) return JF_ERR_UNSUPPORTED;
  if (pool->group_size != 64) return JF_ERR_UNSUPPORTED;
  if (pool->head_dim != 128 && pool->head_dim != 256) return JF_ERR_UNSUPPORTED;
  if (pool->page_size != 64 && pool->page_size != 128 && pool->page_size != 256)
    return JF_ERR_UNSUPPORTED;
  if (pool->num_kv_heads > 65535) return JF_ERR_UNSUPPORTED;
  if (pool->num_pages > 0x7FFFFFFFLL) return JF_ERR_UNSUPPORTED;
  return JF_OK;
}

// Pools of either format, for the entry points that take both (append,
// single-query decode, checkpoint, restore).  TQ4 pools need their codec.
int check_pool_any(const jf_kv_pool* pool) {
  if (!pool || pool->format != JF_FMT_TQ4) return check_pool(pool);
  if (!pool->base || !aligned(pool->base, 16)) return JF_ERR_INVALID_ARG;
  if (pool->num_pages < 1 || pool->num_kv_heads < 1) return JF_ERR_INVALID_ARG;
  if (!pool->tq4) return JF_ERR_INVALID_ARG;
  if (pool->head_dim != 128 && pool->head_dim != 256) return JF_ERR_UNSUPPORTED;
  if (pool->page_size != 64 && pool->page_size != 128 && pool->page_size != 256)
    return JF_ERR_UNSUPPORTED;
  if (pool->num_kv_heads > 65535) return JF_ERR_UNSUPPORTED;
  if (pool->num_pages > 0x7FFFFFFFLL) return JF_ERR_UNSUPPORTED;
  return JF_OK;
}

// Pools of the 8-bit block format.
int check_pool8(const jf_kv_pool* pool) {
  if (!pool || !pool->base || !aligned(pool->base, 16)) return JF_ERR_INVALID_ARG;
  if (pool->num_pages < 1 || pool->num_kv_heads < 1) return JF_ERR_INVALID_ARG;
  if (pool->format != JF_FMT_E4M3_B32) return JF_ERR_UNSUPPORTED;
  if (pool->head_dim != 128 && pool->head_dim != 256) return JF_ERR_UNSUPPORTED;
  if (pool->page_size != 64 && pool->page_size != 128 && pool->page_size != 256)
    return JF_ERR_UNSUPPORTED;
  if (pool->num_kv_heads > 65535) return JF_ERR_UNSUPPORTED;
  if (pool->num_pages > 0x7FFFFFFFLL) return JF_ERR_UNSUPPORTED;
  return JF_OK;
}

// Pools of any format, for the entry points that read or copy all of them
// (single-query decode, prefill; page copies take latent pools as well).
int check_pool_read(const jf_kv_pool* pool) {
  return pool && pool->format == JF_FMT_E4M3_B32 ? check_pool8(pool) : check_pool_any(pool);
}

// Latent pools.
int check_pool_latent(const jf_kv_pool* pool) {
  if (!pool || !pool->base || !aligned(pool->base, 16)) return JF_ERR_INVALID_ARG;
  if (pool->num_pages < 1 || pool->num_kv_heads < 1) return JF_ERR_INVALID_ARG;
  if (pool->format != JF_FMT_LATENT16) return JF_ERR_UNSUPPORTED;
  if (pool->num_kv_heads != 1) return JF_ERR_UNSUPPORTED;
  if (pool->head_dim != 256 + JF_LATENT_ROT && pool->head_dim != 512 + JF_LATENT_ROT)
    return JF_ERR_UNSUPPORTED;
  if (pool->page_size != 64 && pool->page_size != 128 && pool->page_size != 256)
    return JF_ERR_UNSUPPORTED;
  // a row's index is a 32-bit coordinate
  if (pool->num_pages > 0x7FFFFFFFLL / pool->page_size) return JF_ERR_UNSUPPORTED;
  return JF_OK;
}

// What page copies need to know of a pool: its pages' size.
int copy_geom(const jf_kv_pool* pool, Geom* g) {
  const bool latent = pool && pool->format == JF_FMT_LATENT16;
  const int st = latent ? check_pool_latent(pool) : check_pool_read(pool);
  if (st) return st;
  if (latent) {
    *g = Geom{};
    g->num_pages = pool->num_pages;
    g->page_bytes = (int64_t)pool->page_size * pool->head_dim * 2;
  } else {
    *g = make_geom(*pool);
  }
  return JF_OK;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// 5-D map over the code rows of a pool: (byte in row, slot, KV head, K|V, page),
// box = (row bytes, rows_per_box, 1, 1, 1), 128B (or 64B) swizzle.
int make_codes_map(const Geom& g, void* base, int rows_per_box, CUtensorMap* map) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return JF_ERR_CUDA;
  cuuint64_t dims[5] = {(cuuint64_t)g.CB, (cuuint64_t)g.P, (cuuint64_t)g.Hkv, 2,
                        (cuuint64_t)g.num_pages};
  cuuint64_t strides[4] = {(cuuint64_t)g.CB, (cuuint64_t)g.P * g.CB,
                           (cuuint64_t)g.codes_region, (cuuint64_t)g.page_bytes};
  cuuint32_t box[5] = {(cuuint32_t)g.CB, (cuuint32_t)rows_per_box, 1, 1, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  CUtensorMapSwizzle sw = g.CB == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, base, dims, strides, box, estr,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? JF_OK : JF_ERR_CUDA;
}

}  // namespace

namespace jfkv {

// 5-D map over the code rows of an 8-bit pool: (byte of a 128-byte half, half,
// row of K or V over all KV heads, K|V, page), box = (128, halves, rows, kv, 1),
// 128B swizzle.
int kv8_tensor_map(const Geom& g, void* base, int halves, int rows, int kv, CUtensorMap* map) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return JF_ERR_CUDA;
  cuuint64_t dims[5] = {128, (cuuint64_t)g.D / 128, (cuuint64_t)g.Hkv * g.P, 2,
                        (cuuint64_t)g.num_pages};
  cuuint64_t strides[4] = {128, (cuuint64_t)g.D, (cuuint64_t)g.codes_region,
                           (cuuint64_t)g.page_bytes};
  cuuint32_t box[5] = {128, (cuuint32_t)halves, (cuuint32_t)rows, (cuuint32_t)kv, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, base, dims, strides, box, estr,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? JF_OK : JF_ERR_CUDA;
}

// 2-D map over rows of bf16 channels that adjoin, box = 64 channels of box_rows rows, 128B swizzle.
int bf16_rows_map(const void* base, int64_t channels, int64_t rows, int box_rows, CUtensorMap* map) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return JF_ERR_CUDA;
  cuuint64_t dims[2] = {(cuuint64_t)channels, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)channels * 2};
  cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides,
                   box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? JF_OK : JF_ERR_CUDA;
}

// 3-D map over the same rows: (channel of a 64-channel chunk, row, chunk), box = 64 rows of box_chunks
// chunks, which come to lie chunk after chunk.
int bf16_chunks_map(const void* base, int64_t channels, int64_t rows, int box_chunks, CUtensorMap* map) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return JF_ERR_CUDA;
  cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)channels / 64};
  cuuint64_t strides[2] = {(cuuint64_t)channels * 2, 128};
  cuuint32_t box[3] = {64, 64, (cuuint32_t)box_chunks};
  cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides,
                   box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? JF_OK : JF_ERR_CUDA;
}

// 3-D map over queries [C, H, 192], box = 64 channels of 128 queries of a head, 128B swizzle.
int latent_query_map(const void* q, int64_t H, int64_t C, CUtensorMap* map) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return JF_ERR_CUDA;
  const cuuint64_t row = 128 + JF_LATENT_ROT;
  cuuint64_t dims[3] = {row, (cuuint64_t)H, (cuuint64_t)C};
  cuuint64_t strides[2] = {row * 2, row * 2 * (cuuint64_t)H};
  cuuint32_t box[3] = {64, 1, 128};
  cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box,
                   estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv

extern "C" {

size_t jf_kv_page_bytes(int32_t num_kv_heads, int32_t page_size, int32_t head_dim) {
  if (num_kv_heads < 1 || page_size < 1 || (head_dim != 128 && head_dim != 256)) return 0;
  jf_kv_pool p{};
  p.num_pages = 1;
  p.page_size = page_size;
  p.num_kv_heads = num_kv_heads;
  p.head_dim = head_dim;
  return (size_t)make_geom(p).page_bytes;
}

size_t jf_kv_page_bytes_fmt(int32_t format, int32_t num_kv_heads, int32_t page_size,
                            int32_t head_dim) {
  if (format == JF_FMT_LATENT16) {
    if (num_kv_heads != 1 || page_size < 1) return 0;
    if (head_dim != 256 + JF_LATENT_ROT && head_dim != 512 + JF_LATENT_ROT) return 0;
    return (size_t)page_size * head_dim * 2;
  }
  if (format != JF_FMT_AFFINE4_G64 && format != JF_FMT_TQ4 && format != JF_FMT_E4M3_B32) return 0;
  if (format == JF_FMT_E4M3_B32 && page_size % 32) return 0;
  if (num_kv_heads < 1 || page_size < 1 || (head_dim != 128 && head_dim != 256)) return 0;
  jf_kv_pool p{};
  p.num_pages = 1;
  p.page_size = page_size;
  p.num_kv_heads = num_kv_heads;
  p.head_dim = head_dim;
  p.format = format;
  return (size_t)make_geom(p).page_bytes;
}

int jf_tq4_codebook(int32_t head_dim, float* centroids) {
  if (!centroids || head_dim < 3 || head_dim > 65536) return JF_ERR_INVALID_ARG;
  return tq4_codebook_host(head_dim, centroids);
}

size_t jf_attn_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                               int32_t head_dim, int32_t num_splits) {
  if (batch < 1 || num_q_heads < 1 || num_kv_heads < 1 || num_splits < 1) return 0;
  if (num_q_heads % num_kv_heads) return 0;
  if (head_dim != 128 && head_dim != 256) return 0;
  return decode_workspace_bytes(batch, num_q_heads, head_dim, num_splits);
}

size_t jf_prefill_workspace_bytes(void) { return 256; }

int jf_kv_quantize_append(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                          int32_t num_requests, const int32_t* row_req, const int32_t* row_pos,
                          const void* k, const void* v, int32_t n_rows, int32_t* err_flag,
                          void* stream) {
  int st = check_pool_any(pool);
  if (st) return st;
  if (n_rows < 0 || pt_stride < 1 || num_requests < 1) return JF_ERR_INVALID_ARG;
  if (n_rows == 0) return JF_OK;
  if (!page_table || !row_req || !row_pos || !k || !v) return JF_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16)) return JF_ERR_INVALID_ARG;
  const Geom g = make_geom(*pool);
  if (pool->format == JF_FMT_TQ4) {
    Tq4Params prm;
    st = tq4_make_params(pool->tq4, g.D, &prm);
    if (st) return st;
    return launch_tq4_append(g, *pool, prm, page_table, pt_stride, num_requests, row_req,
                             row_pos, k, v, n_rows, err_flag, static_cast<cudaStream_t>(stream));
  }
  return launch_append(g, *pool, page_table, pt_stride, num_requests, row_req, row_pos, k, v,
                       n_rows, err_flag, static_cast<cudaStream_t>(stream));
}

static int decode_common(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                         const int32_t* context_lens, int32_t batch, const void* k_new,
                         const void* v_new, const void* q, int32_t num_q_heads,
                         float softmax_scale, void* out, void* workspace, size_t workspace_bytes,
                         int32_t num_splits, void* stream, int32_t q_len = 1) {
  const bool kv8 = pool && pool->format == JF_FMT_E4M3_B32;
  if (kv8 && (q_len != 1 || k_new)) return JF_ERR_UNSUPPORTED;   // single-query decode only
  int st = check_pool_read(pool);
  if (st) return st;
  if (!page_table || !context_lens || !q || !out || !workspace) return JF_ERR_INVALID_ARG;
  if (batch < 1 || batch > 65535 || pt_stride < 1 || num_q_heads < 1) return JF_ERR_INVALID_ARG;
  if (num_q_heads % pool->num_kv_heads) return JF_ERR_INVALID_ARG;
  if (num_q_heads / pool->num_kv_heads > 8) return JF_ERR_UNSUPPORTED;
  if (num_splits < 1 || num_splits > 65535) return JF_ERR_INVALID_ARG;
  if (q_len < 1 || q_len > 4) return JF_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256)) return JF_ERR_INVALID_ARG;
  if (k_new && (!aligned(k_new, 16) || !aligned(v_new, 16))) return JF_ERR_INVALID_ARG;
  const size_t need = jf_attn_workspace_bytes(batch, q_len * num_q_heads, pool->num_kv_heads,
                                              pool->head_dim, num_splits);
  if (workspace_bytes < need) return JF_ERR_WORKSPACE_TOO_SMALL;
  const Geom g = make_geom(*pool);
  if (kv8) {
    CUtensorMap tmap8;
    st = kv8_tensor_map(g, pool->base, g.D / 128, kv8_box_rows(), 2, &tmap8);
    if (st) return st;
    return launch_kv8_decode(g, *pool, tmap8, page_table, pt_stride, context_lens, batch, q,
                             num_q_heads, softmax_scale, out, workspace, num_splits, nullptr,
                             nullptr, nullptr, 0, static_cast<cudaStream_t>(stream));
  }
  Tq4Params prm;
  if (pool->format == JF_FMT_TQ4) {
    st = tq4_make_params(pool->tq4, g.D, &prm);
    if (st) return st;
  }
  CUtensorMap tmap;
  st = make_codes_map(g, pool->base, decode_box_rows(), &tmap);
  if (st) return st;
  if (pool->format == JF_FMT_TQ4) {
    return launch_tq4_decode(g, *pool, tmap, prm, page_table, pt_stride, context_lens, batch, q,
                             num_q_heads, softmax_scale, out, workspace, num_splits,
                             static_cast<cudaStream_t>(stream), k_new, v_new, q_len);
  }
  return launch_decode(g, *pool, tmap, page_table, pt_stride, context_lens, batch, q,
                       num_q_heads, softmax_scale, out, workspace, num_splits,
                       static_cast<cudaStream_t>(stream), k_new, v_new, q_len);
}

int jf_paged_decode_attn(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                         const int32_t* context_lens, int32_t batch, const void* q,
                         int32_t num_q_heads, float softmax_scale, void* out, void* workspace,
                         size_t workspace_bytes, int32_t num_splits, void* stream) {
  return decode_common(pool, page_table, pt_stride, context_lens, batch, nullptr, nullptr, q,
                       num_q_heads, softmax_scale, out, workspace, workspace_bytes, num_splits,
                       stream);
}

int jf_paged_verify_attn(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                         const int32_t* context_lens, int32_t batch, const void* q,
                         int32_t q_len, int32_t num_q_heads, float softmax_scale, void* out,
                         void* workspace, size_t workspace_bytes, int32_t num_splits,
                         void* stream) {
  if (q_len < 1 || q_len > 4) return JF_ERR_INVALID_ARG;
  if (pool && pool->format == JF_FMT_E4M3_B32) return JF_ERR_UNSUPPORTED;
  return decode_common(pool, page_table, pt_stride, context_lens, batch, nullptr, nullptr, q,
                       num_q_heads, softmax_scale, out, workspace, workspace_bytes, num_splits,
                       stream, q_len);
}

int jf_paged_decode_append_attn(const jf_kv_pool* pool, const int32_t* page_table,
                                int32_t pt_stride, const int32_t* context_lens, int32_t batch,
                                const void* k_new, const void* v_new, const void* q,
                                int32_t num_q_heads, float softmax_scale, void* out,
                                void* workspace, size_t workspace_bytes, int32_t num_splits,
                                void* stream) {
  if (!k_new || !v_new) return JF_ERR_INVALID_ARG;
  return decode_common(pool, page_table, pt_stride, context_lens, batch, k_new, v_new, q,
                       num_q_heads, softmax_scale, out, workspace, workspace_bytes, num_splits,
                       stream);
}

}  // extern "C"

namespace {

// The prefill kernel's geometry: 128 MMA rows per CTA (128 / G queries), two
// CTAs per pair, one CTA per SM, 64-position history tiles.
constexpr int64_t kPfRows = 128;
constexpr int64_t kPfTile = 64;

// Wave balance of one chunk over a long prefix (q_start >= 4 chunk_len, so
// its CTA pairs carry nearly equal work W, the prefix's history tiles).
// Pairs run num_sms / 2 at a time.  When the last wave would be partly
// empty, the query tiles that fill it become a tail: the head's pairs run as
// whole waves, and the tail's history is split k ways, so the tail costs
// ceil(pieces / slots) rounds of W / k instead of one more W.  The estimate
// adds a fixed cost for the split launch and its merge and a cost per round
// (0.07 W + 0.03 W per round, fitted on a 2,048-query chunk after 30,720
// positions at 24 / 4 heads, D = 256); the smallest k within 0.05 W of the
// best is taken, only if it beats the unsplit tail by 0.05 W and leaves
// every piece 8 history tiles or more.  head = chunk_len, k = 1: one launch.
struct PfTailPlan {
  int32_t head, k;
};

PfTailPlan prefill_tail_plan(int64_t G, int64_t Hkv, int64_t q_start, int64_t chunk_len,
                             int64_t num_sms) {
  PfTailPlan p{(int32_t)chunk_len, 1};
  if (G < 1 || G > kPfRows || Hkv < 1 || num_sms < 2 || chunk_len < 1 || q_start < 4 * chunk_len)
    return p;
  const int64_t slots = num_sms / 2;
  const int64_t qpp = 2 * (kPfRows / G);                // queries per CTA pair
  const int64_t pph = (chunk_len + qpp - 1) / qpp;      // pairs per KV head
  const int64_t rem = (pph * Hkv) % slots;
  if (pph * Hkv <= slots || rem == 0) return p;
  const int64_t t_tail = (rem + Hkv - 1) / Hkv;         // tail pairs per KV head
  if (t_tail >= pph) return p;
  const int64_t c_head = (pph - t_tail) * qpp;
  const int64_t min_tiles = (q_start + c_head + kPfTile) / kPfTile;   // first tail query's
  double est[9] = {0};
  double best = 1e30;
  for (int s = 2; s <= 8 && min_tiles / s >= 8; ++s) {
    const int64_t rounds = (t_tail * Hkv * s + slots - 1) / slots;
    est[s] = (double)rounds / s + 0.07 + 0.03 * (double)rounds;
    if (est[s] < best) best = est[s];
  }
  if (best > 0.95) return p;
  for (int s = 2; s <= 8; ++s)
    if (est[s] > 0 && est[s] <= best + 0.05) return PfTailPlan{(int32_t)c_head, s};
  return p;
}

// Workspace of the balanced form: the head launch (unsplit) and the tail
// launch (k splits) run one after the other on the same workspace.
size_t prefill_tail_workspace(const PfTailPlan& p, int64_t chunk_len, int64_t Hq, int64_t D,
                              int fmt) {
  const size_t h = prefill_workspace_bytes(p.head, Hq, D, 1, fmt);
  const size_t t = prefill_workspace_bytes(chunk_len - p.head, Hq, D, p.k, fmt);
  return h > t ? h : t;
}

}  // namespace

extern "C" {

size_t jf_prefill_chunk_workspace_bytes(const jf_kv_pool* pool, int32_t q_start,
                                        int32_t chunk_len, int32_t num_q_heads, int32_t num_sms) {
  if (check_pool_read(pool)) return 0;
  if (q_start < 0 || chunk_len < 0 || num_q_heads < 1 || num_sms < 0) return 0;
  if (num_q_heads % pool->num_kv_heads) return 0;
  const bool tq = pool->format == JF_FMT_TQ4;
  const size_t one = tq ? prefill_workspace_bytes(chunk_len, num_q_heads, pool->head_dim, 1,
                                                  JF_FMT_TQ4)
                        : jf_prefill_workspace_bytes();
  if (pool->format == JF_FMT_E4M3_B32) {
    size_t bytes = one;
    for (int causal = 0; causal < 2; ++causal) {
      P8Plan plan;
      kv8_prefill_plan(num_q_heads / pool->num_kv_heads, pool->num_kv_heads, q_start, chunk_len,
                       causal != 0, num_sms ? num_sms : sm_count(), &plan);
      const size_t n = prefill_workspace_bytes(plan.rows, num_q_heads, pool->head_dim, plan.k,
                                               pool->format);
      if (plan.n && n > bytes) bytes = n;
    }
    return bytes;
  }
  const PfTailPlan p = prefill_tail_plan(num_q_heads / pool->num_kv_heads, pool->num_kv_heads,
                                         q_start, chunk_len, num_sms ? num_sms : sm_count());
  if (p.k == 1) return one;
  const size_t bal = prefill_tail_workspace(p, chunk_len, num_q_heads, pool->head_dim,
                                            pool->format);
  return bal > one ? bal : one;
}

int jf_prefill_chunk_attn(const jf_kv_pool* pool, const int32_t* page_table_row, const void* q,
                          int32_t q_start, int32_t chunk_len, int32_t num_q_heads,
                          float softmax_scale, int32_t causal, void* out, void* workspace,
                          size_t workspace_bytes, void* stream) {
  int st = check_pool_read(pool);
  if (st) return st;
  if (!page_table_row || !q || !out || !workspace) return JF_ERR_INVALID_ARG;
  if (q_start < 0 || chunk_len < 0 || num_q_heads < 1) return JF_ERR_INVALID_ARG;
  if (num_q_heads % pool->num_kv_heads) return JF_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  const bool tq = pool->format == JF_FMT_TQ4;
  const size_t need = tq ? prefill_workspace_bytes(chunk_len, num_q_heads, pool->head_dim, 1,
                                                   JF_FMT_TQ4)
                         : jf_prefill_workspace_bytes();
  if (workspace_bytes < need) return JF_ERR_WORKSPACE_TOO_SMALL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, tq ? 256 : 16))
    return JF_ERR_INVALID_ARG;
  if ((int64_t)q_start + chunk_len > 0x7FFFFFFF) return JF_ERR_INVALID_ARG;
  if (chunk_len == 0) return JF_OK;
  const Geom g = make_geom(*pool);
  if (num_q_heads / pool->num_kv_heads > 128) return JF_ERR_UNSUPPORTED;
  Tq4Params prm;
  if (tq) {
    st = tq4_make_params(pool->tq4, g.D, &prm);
    if (st) return st;
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int64_t row0 = 0;
  if (pool->format == JF_FMT_E4M3_B32) {
    P8Plan plan;
    kv8_prefill_plan(num_q_heads / pool->num_kv_heads, pool->num_kv_heads, q_start, chunk_len,
                     causal != 0, sm_count(), &plan);
    const bool planned =
        plan.n > 0 && aligned(workspace, 256) &&
        workspace_bytes >= prefill_workspace_bytes(plan.rows, num_q_heads, g.D, plan.k, pool->format);
    return launch_prefill_batch(g, *pool, &page_table_row, &q_start, &chunk_len, q, &row0, 1,
                                num_q_heads, softmax_scale, causal, out, workspace, s,
                                planned ? plan.k : 1, planned ? plan.rows : chunk_len, nullptr,
                                planned ? &plan : nullptr);
  }
  const PfTailPlan p = prefill_tail_plan(num_q_heads / pool->num_kv_heads, pool->num_kv_heads,
                                         q_start, chunk_len, sm_count());
  if (p.k > 1 && aligned(workspace, 256) &&
      workspace_bytes >= prefill_tail_workspace(p, chunk_len, num_q_heads, g.D, pool->format)) {
    // the head's query tiles as whole waves, then the tail's with split histories
    const size_t row_bytes = (size_t)num_q_heads * g.D * 2;
    const int32_t t_start = q_start + p.head, t_len = chunk_len - p.head;
    const void* q_t = static_cast<const uint8_t*>(q) + (size_t)p.head * row_bytes;
    void* out_t = static_cast<uint8_t*>(out) + (size_t)p.head * row_bytes;
    st = launch_prefill_batch(g, *pool, &page_table_row, &q_start, &p.head, q, &row0, 1,
                              num_q_heads, softmax_scale, causal, out, workspace, s, 1, p.head,
                              tq ? &prm : nullptr);
    if (st) return st;
    return launch_prefill_batch(g, *pool, &page_table_row, &t_start, &t_len, q_t, &row0, 1,
                                num_q_heads, softmax_scale, causal, out_t, workspace, s, p.k,
                                t_len, tq ? &prm : nullptr);
  }
  if (tq)
    return launch_prefill_batch(g, *pool, &page_table_row, &q_start, &chunk_len, q, &row0, 1,
                                num_q_heads, softmax_scale, causal, out, workspace, s, 1,
                                chunk_len, &prm);
  CUtensorMap tmap{};
  return launch_prefill(g, *pool, tmap, page_table_row, q, q_start, chunk_len, num_q_heads,
                        softmax_scale, causal, out, workspace, s);
}

size_t jf_prefill_batch_workspace_bytes(int32_t format, int64_t total_rows, int32_t num_q_heads,
                                        int32_t head_dim, int32_t num_splits) {
  if (format != JF_FMT_AFFINE4_G64 && format != JF_FMT_TQ4 && format != JF_FMT_E4M3_B32) return 0;
  if (total_rows < 0 || num_q_heads < 1 || num_splits < 1 || num_splits > 65535) return 0;
  if (head_dim != 128 && head_dim != 256) return 0;
  return prefill_workspace_bytes(total_rows, num_q_heads, head_dim, num_splits, format);
}

int jf_prefill_batch_attn(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                          int32_t batch, const int32_t* q_start, const int32_t* chunk_len,
                          const void* q, int32_t num_q_heads, float softmax_scale, int32_t causal,
                          int32_t num_splits, void* out, void* workspace, size_t workspace_bytes,
                          void* stream) {
  int st = check_pool_read(pool);
  if (st) return st;
  if (batch < 1 || pt_stride < 1 || num_q_heads < 1) return JF_ERR_INVALID_ARG;
  if (batch > JF_PREFILL_MAX_BATCH) return JF_ERR_UNSUPPORTED;
  if (!page_table || !q_start || !chunk_len || !q || !out || !workspace) return JF_ERR_INVALID_ARG;
  if (num_q_heads % pool->num_kv_heads) return JF_ERR_INVALID_ARG;
  if (num_q_heads / pool->num_kv_heads > 128) return JF_ERR_UNSUPPORTED;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  if (num_splits < 1 || num_splits > 65535) return JF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256)) return JF_ERR_INVALID_ARG;
  const int32_t* rows[JF_PREFILL_MAX_BATCH];
  int64_t row0[JF_PREFILL_MAX_BATCH];
  int64_t acc = 0;
  for (int b = 0; b < batch; ++b) {
    if (q_start[b] < 0 || chunk_len[b] < 0) return JF_ERR_INVALID_ARG;
    if ((int64_t)q_start[b] + chunk_len[b] > (int64_t)pt_stride * pool->page_size)
      return JF_ERR_INVALID_ARG;   // the chunk must fit the request's page-table row
    rows[b] = page_table + (int64_t)b * pt_stride;
    row0[b] = acc;
    acc += chunk_len[b];
  }
  if (acc > 0x7FFFFFFF) return JF_ERR_INVALID_ARG;
  if (workspace_bytes <
      prefill_workspace_bytes(acc, num_q_heads, pool->head_dim, num_splits, pool->format))
    return JF_ERR_WORKSPACE_TOO_SMALL;
  if (acc == 0) return JF_OK;
  const Geom g = make_geom(*pool);
  Tq4Params prm;
  if (pool->format == JF_FMT_TQ4) {
    st = tq4_make_params(pool->tq4, g.D, &prm);
    if (st) return st;
  }
  return launch_prefill_batch(g, *pool, rows, q_start, chunk_len, q, row0, batch, num_q_heads,
                              softmax_scale, causal, out, workspace,
                              static_cast<cudaStream_t>(stream), num_splits, acc,
                              pool->format == JF_FMT_TQ4 ? &prm : nullptr);
}

int64_t jf_reservation_pages(int64_t prompt_len, int64_t output_len, int64_t g_out,
                             int32_t page_size) {
  if (prompt_len < 0 || output_len < 0 || g_out < 0 || page_size < 1) return -1;
  const int64_t out = output_len < g_out ? output_len : g_out;
  if (prompt_len > INT64_MAX - out - page_size) return -1;
  return (prompt_len + out + page_size - 1) / page_size;
}

int jf_kv_checkpoint(const jf_kv_pool* pool, const int32_t* page_table_row, int32_t num_pages,
                     void* dst, size_t dst_bytes, int32_t* err_flag, void* stream) {
  Geom g;
  const int st = copy_geom(pool, &g);
  if (st) return st;
  if (num_pages < 0) return JF_ERR_INVALID_ARG;
  if (num_pages == 0) return JF_OK;
  if (!page_table_row || !dst || !aligned(dst, 16)) return JF_ERR_INVALID_ARG;
  if (dst_bytes < (size_t)num_pages * (size_t)g.page_bytes) return JF_ERR_INVALID_ARG;
  return launch_page_copy(g, *pool, page_table_row, num_pages, dst, err_flag, true,
                          static_cast<cudaStream_t>(stream));
}

int jf_kv_restore(const jf_kv_pool* pool, const int32_t* page_table_row, int32_t num_pages,
                  const void* src, size_t src_bytes, int32_t* err_flag, void* stream) {
  Geom g;
  const int st = copy_geom(pool, &g);
  if (st) return st;
  if (num_pages < 0) return JF_ERR_INVALID_ARG;
  if (num_pages == 0) return JF_OK;
  if (!page_table_row || !src || !aligned(src, 16)) return JF_ERR_INVALID_ARG;
  if (src_bytes < (size_t)num_pages * (size_t)g.page_bytes) return JF_ERR_INVALID_ARG;
  return launch_page_copy(g, *pool, page_table_row, num_pages, const_cast<void*>(src), err_flag,
                          false, static_cast<cudaStream_t>(stream));
}

// ---------------------------------------------------------------------------
// Rotary axes and the 8-bit block-scaled cache
// ---------------------------------------------------------------------------
int jf_rope_axes(const jf_rope* rope, const int32_t* positions, int64_t pos_stride,
                 int32_t n_tokens, int32_t head_dim, const jf_rope_rows* q, const jf_rope_rows* k,
                 int32_t dtype, int32_t inverse, void* stream) {
  if (!rope || !q || !k) return JF_ERR_INVALID_ARG;
  if (dtype != JF_DTYPE_BF16 && dtype != JF_DTYPE_F16 && dtype != JF_DTYPE_F32)
    return JF_ERR_UNSUPPORTED;
  if (rope->pairing != JF_ROPE_PAIR_HALF && rope->pairing != JF_ROPE_PAIR_ADJACENT)
    return JF_ERR_INVALID_ARG;
  if (rope->num_axes < 1 || rope->num_axes > JF_ROPE_MAX_AXES) return JF_ERR_INVALID_ARG;
  if (rope->rotary_dim < 16 || rope->rotary_dim % 16 || rope->rotary_dim > 256)
    return JF_ERR_UNSUPPORTED;
  if (head_dim < rope->rotary_dim || head_dim % 16 || head_dim > 512) return JF_ERR_UNSUPPORTED;
  for (int i = 0; i < rope->rotary_dim / 2; ++i) {
    if (!(rope->inv_freq[i] > -4294967296.f && rope->inv_freq[i] < 4294967296.f))
      return JF_ERR_INVALID_ARG;
    if (rope->axis[i] >= rope->num_axes) return JF_ERR_INVALID_ARG;
  }
  if (n_tokens < 0 || pos_stride < 0) return JF_ERR_INVALID_ARG;
  const int64_t vec = dtype == JF_DTYPE_F32 ? 4 : 8;   // elements of 16 bytes
  const jf_rope_rows* rows[2] = {q, k};
  for (const jf_rope_rows* r : rows) {
    if (r->num_heads < 0 || r->num_heads > 65535) return JF_ERR_INVALID_ARG;
    if (r->num_heads == 0 || n_tokens == 0) continue;
    if (!r->in || !r->out || !aligned(r->in, 16) || !aligned(r->out, 16)) return JF_ERR_INVALID_ARG;
    if (r->in_token_stride % vec || r->in_head_stride % vec || r->out_token_stride % vec ||
        r->out_head_stride % vec)
      return JF_ERR_INVALID_ARG;
    if (r->in == r->out && (r->in_token_stride != r->out_token_stride ||
                            r->in_head_stride != r->out_head_stride))
      return JF_ERR_INVALID_ARG;   // in place, but to other rows
  }
  if (n_tokens == 0 || q->num_heads + k->num_heads == 0) return JF_OK;
  if (!positions) return JF_ERR_INVALID_ARG;
  return launch_rope(*rope, positions, pos_stride, n_tokens, head_dim, *q, *k, dtype, inverse,
                     static_cast<cudaStream_t>(stream));
}

static int kv8_rows(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                    int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                    void* k, int64_t k_stride, void* v, int64_t v_stride, int32_t n_rows,
                    int32_t* err_flag, bool read, void* stream) {
  int st = check_pool8(pool);
  if (st) return st;
  if (n_rows < 0 || pt_stride < 1 || num_requests < 1) return JF_ERR_INVALID_ARG;
  if (n_rows == 0) return JF_OK;
  if (!page_table || !start_pos || !row_offsets || !k || !v) return JF_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16)) return JF_ERR_INVALID_ARG;
  const int64_t row = (int64_t)pool->num_kv_heads * pool->head_dim;
  if (k_stride % 8 || v_stride % 8 || k_stride < row || v_stride < row) return JF_ERR_INVALID_ARG;
  const Geom g = make_geom(*pool);
  return launch_kv8_rows(g, *pool, page_table, pt_stride, num_requests, start_pos, row_offsets, k,
                         k_stride, v, v_stride, n_rows, err_flag, read,
                         static_cast<cudaStream_t>(stream));
}

int jf_kv8_append(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                  int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                  const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  int32_t n_rows, int32_t* err_flag, void* stream) {
  return kv8_rows(pool, page_table, pt_stride, num_requests, start_pos, row_offsets,
                  const_cast<void*>(k), k_stride, const_cast<void*>(v), v_stride, n_rows, err_flag,
                  false, stream);
}

int jf_kv8_read(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                void* k, int64_t k_stride, void* v, int64_t v_stride, int32_t n_rows,
                int32_t* err_flag, void* stream) {
  return kv8_rows(pool, page_table, pt_stride, num_requests, start_pos, row_offsets, k, k_stride,
                  v, v_stride, n_rows, err_flag, true, stream);
}

size_t jf_decode_weights_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                         int32_t head_dim, int32_t num_splits,
                                         int64_t weight_stride) {
  if (weight_stride < 1 || weight_stride > 0x7FFFFFFF) return 0;
  const size_t n = jf_attn_workspace_bytes(batch, num_q_heads, num_kv_heads, head_dim, num_splits);
  if (n == 0) return 0;
  return (n + 255) / 256 * 256 +
         (size_t)batch * num_kv_heads *
             (size_t)kv8_score_floats(num_q_heads / num_kv_heads, weight_stride) * 4;
}

int jf_paged_decode_weights_attn(const jf_kv_pool* pool, const int32_t* page_table,
                                 int32_t pt_stride, const int32_t* context_lens, int32_t batch,
                                 const void* q, int32_t num_q_heads, float softmax_scale,
                                 void* out, const float* weights_in, float* weights_out,
                                 int64_t weight_stride, void* workspace, size_t workspace_bytes,
                                 int32_t num_splits, void* stream) {
  int st = check_pool8(pool);
  if (st) return st;
  if (!page_table || !context_lens || !q || !out || !weights_out || !workspace)
    return JF_ERR_INVALID_ARG;
  if (batch < 1 || batch > 65535 || pt_stride < 1 || num_q_heads < 1) return JF_ERR_INVALID_ARG;
  if (num_q_heads % pool->num_kv_heads) return JF_ERR_INVALID_ARG;
  if (num_q_heads / pool->num_kv_heads > 8) return JF_ERR_UNSUPPORTED;
  if (num_splits < 1 || num_splits > 65535) return JF_ERR_INVALID_ARG;
  if (weight_stride < 1 || weight_stride > 0x7FFFFFFF) return JF_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) ||
      !aligned(weights_in, 4) || !aligned(weights_out, 4))
    return JF_ERR_INVALID_ARG;
  const size_t base = (jf_attn_workspace_bytes(batch, num_q_heads, pool->num_kv_heads,
                                               pool->head_dim, num_splits) + 255) / 256 * 256;
  if (workspace_bytes < jf_decode_weights_workspace_bytes(batch, num_q_heads, pool->num_kv_heads,
                                                          pool->head_dim, num_splits,
                                                          weight_stride))
    return JF_ERR_WORKSPACE_TOO_SMALL;
  const Geom g = make_geom(*pool);
  CUtensorMap tmap;
  st = kv8_tensor_map(g, pool->base, g.D / 128, kv8_box_rows(), 2, &tmap);
  if (st) return st;
  return launch_kv8_decode(g, *pool, tmap, page_table, pt_stride, context_lens, batch, q,
                           num_q_heads, softmax_scale, out, workspace, num_splits,
                           reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + base),
                           weights_in, weights_out, weight_stride,
                           static_cast<cudaStream_t>(stream));
}

int jf_kv8_evict(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                 const int32_t* context_lens, int32_t batch, const float* weights,
                 int64_t weight_stride, int32_t budget, int32_t sinks, int32_t recent,
                 const int32_t* dst_page_table, int32_t dst_stride, int32_t* dst_context_lens,
                 float* dst_weights, int32_t* kept, int32_t* err_flag, void* stream) {
  const int st = check_pool8(pool);
  if (st) return st;
  if (!page_table || !context_lens || !weights || !dst_page_table || !dst_context_lens || !kept)
    return JF_ERR_INVALID_ARG;
  if (batch < 1 || batch > 65535 || pt_stride < 1 || dst_stride < 1) return JF_ERR_INVALID_ARG;
  if (weight_stride < 1 || weight_stride > 0x7FFFFFFF) return JF_ERR_INVALID_ARG;
  if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
    return JF_ERR_INVALID_ARG;
  if (!aligned(weights, 4) || !aligned(dst_weights, 4)) return JF_ERR_INVALID_ARG;
  const Geom g = make_geom(*pool);
  return launch_kv8_evict(g, *pool, page_table, pt_stride, context_lens, batch, weights,
                          weight_stride, budget, sinks, recent, dst_page_table, dst_stride,
                          dst_context_lens, dst_weights, kept, err_flag,
                          static_cast<cudaStream_t>(stream));
}

// ---------------------------------------------------------------------------
// The latent cache
// ---------------------------------------------------------------------------
static int latent_rows(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                       int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                       void* latent, int64_t latent_stride, void* k_rot, int64_t rot_stride,
                       int32_t n_rows, int32_t* err_flag, bool read, void* stream) {
  const int st = check_pool_latent(pool);
  if (st) return st;
  if (n_rows < 0 || pt_stride < 1 || num_requests < 1) return JF_ERR_INVALID_ARG;
  if (n_rows == 0) return JF_OK;
  if (!page_table || !start_pos || !row_offsets || !latent || !k_rot) return JF_ERR_INVALID_ARG;
  if (!aligned(latent, 16) || !aligned(k_rot, 16)) return JF_ERR_INVALID_ARG;
  if (latent_stride % 8 || rot_stride % 8 || latent_stride < pool->head_dim - JF_LATENT_ROT ||
      rot_stride < JF_LATENT_ROT)
    return JF_ERR_INVALID_ARG;
  return launch_latent_rows(latent_pool(*pool), page_table, pt_stride, num_requests, start_pos,
                            row_offsets, latent, latent_stride, k_rot, rot_stride, n_rows,
                            err_flag, read, static_cast<cudaStream_t>(stream));
}

int jf_latent_append(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                     int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                     const void* latent, int64_t latent_stride, const void* k_rot,
                     int64_t rot_stride, int32_t n_rows, int32_t* err_flag, void* stream) {
  return latent_rows(pool, page_table, pt_stride, num_requests, start_pos, row_offsets,
                     const_cast<void*>(latent), latent_stride, const_cast<void*>(k_rot),
                     rot_stride, n_rows, err_flag, false, stream);
}

int jf_latent_read(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                   int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                   void* latent, int64_t latent_stride, void* k_rot, int64_t rot_stride,
                   int32_t n_rows, int32_t* err_flag, void* stream) {
  return latent_rows(pool, page_table, pt_stride, num_requests, start_pos, row_offsets, latent,
                     latent_stride, k_rot, rot_stride, n_rows, err_flag, true, stream);
}

size_t jf_latent_workspace_bytes(int32_t batch, int32_t num_heads, int32_t latent_dim,
                                 int32_t num_groups, int32_t num_sms) {
  if (batch < 1 || batch > 65535 || num_heads < 1 || num_heads > 1024) return 0;
  if (latent_dim != 256 && latent_dim != 512) return 0;
  if (num_groups < 0 || num_groups > JF_LATENT_MAX_GROUPS || num_sms < 0) return 0;
  return latent_decode_workspace_bytes(batch, num_heads, latent_dim, num_groups,
                                       num_sms ? num_sms : sm_count());
}

static int latent_decode(const jf_kv_pool* pool, const int32_t* prefix_table,
                         int32_t prefix_stride, const int32_t* prefix_lens,
                         const int32_t* group_offsets, int32_t num_groups,
                         const int32_t* page_table, int32_t pt_stride,
                         const int32_t* context_lens, int32_t batch, const void* q,
                         int32_t num_heads, float softmax_scale, void* out, void* workspace,
                         size_t workspace_bytes, void* stream) {
  const int st = check_pool_latent(pool);
  if (st) return st;
  if (!page_table || !context_lens || !q || !out || !workspace) return JF_ERR_INVALID_ARG;
  if (batch < 1 || batch > 65535 || pt_stride < 1 || num_heads < 1) return JF_ERR_INVALID_ARG;
  if (num_heads > 1024) return JF_ERR_UNSUPPORTED;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256)) return JF_ERR_INVALID_ARG;
  LatentDecode a{};
  if (num_groups) {
    if (!prefix_table || !prefix_lens || !group_offsets || prefix_stride < 1 || num_groups < 1)
      return JF_ERR_INVALID_ARG;
    if (num_groups > JF_LATENT_MAX_GROUPS) return JF_ERR_UNSUPPORTED;
    if (group_offsets[0] != 0 || group_offsets[num_groups] != batch) return JF_ERR_INVALID_ARG;
    for (int g = 0; g < num_groups; ++g)
      if (group_offsets[g + 1] < group_offsets[g]) return JF_ERR_INVALID_ARG;
    for (int g = 0; g <= num_groups; ++g) a.first[g] = group_offsets[g];
  }
  if (workspace_bytes < jf_latent_workspace_bytes(batch, num_heads, pool->head_dim - JF_LATENT_ROT,
                                                  num_groups, 0))
    return JF_ERR_WORKSPACE_TOO_SMALL;
  a.pool = latent_pool(*pool);
  a.prefix_table = prefix_table;
  a.prefix_lens = prefix_lens;
  a.prefix_stride = prefix_stride;
  a.num_groups = num_groups;
  a.page_table = page_table;
  a.context_lens = context_lens;
  a.pt_stride = pt_stride;
  a.batch = batch;
  a.H = num_heads;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  a.status = static_cast<int32_t*>(workspace);
  return launch_latent_decode(a, workspace, static_cast<cudaStream_t>(stream));
}

int jf_latent_decode_attn(const jf_kv_pool* pool, const int32_t* page_table, int32_t pt_stride,
                          const int32_t* context_lens, int32_t batch, const void* q,
                          int32_t num_heads, float softmax_scale, void* out, void* workspace,
                          size_t workspace_bytes, void* stream) {
  return latent_decode(pool, nullptr, 0, nullptr, nullptr, 0, page_table, pt_stride, context_lens,
                       batch, q, num_heads, softmax_scale, out, workspace, workspace_bytes, stream);
}

int jf_latent_prefix_decode_attn(const jf_kv_pool* pool, const int32_t* prefix_table,
                                 int32_t prefix_stride, const int32_t* prefix_lens,
                                 const int32_t* group_offsets, int32_t num_groups,
                                 const int32_t* page_table, int32_t pt_stride,
                                 const int32_t* context_lens, int32_t batch, const void* q,
                                 int32_t num_heads, float softmax_scale, void* out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (num_groups < 1) return JF_ERR_INVALID_ARG;
  return latent_decode(pool, prefix_table, prefix_stride, prefix_lens, group_offsets, num_groups,
                       page_table, pt_stride, context_lens, batch, q, num_heads, softmax_scale,
                       out, workspace, workspace_bytes, stream);
}

size_t jf_latent_prefill_workspace_bytes(int32_t q_start, int32_t chunk_len, int32_t num_heads,
                                         int32_t num_sms) {
  if (q_start < 0 || chunk_len < 0 || num_heads < 1 || num_heads > 1024 || num_sms < 0) return 0;
  if ((int64_t)q_start + chunk_len > JF_LATENT_MAX_POSITIONS) return 0;
  return latent_prefill_workspace_bytes(q_start, chunk_len, num_heads,
                                        num_sms ? num_sms : sm_count());
}

int jf_latent_prefill_attn(const jf_kv_pool* pool, const int32_t* page_table_row, const void* q,
                           int32_t q_start, int32_t chunk_len, int32_t num_heads,
                           const void* w_k, const void* w_v, float softmax_scale, int32_t causal,
                           void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = check_pool_latent(pool);
  if (st) return st;
  if (q_start < 0 || chunk_len < 0 || num_heads < 1) return JF_ERR_INVALID_ARG;
  if (num_heads > 1024) return JF_ERR_UNSUPPORTED;
  if ((int64_t)q_start + chunk_len > JF_LATENT_MAX_POSITIONS) return JF_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  if (chunk_len == 0) return JF_OK;
  if (!page_table_row || !q || !w_k || !w_v || !out || !workspace) return JF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(w_k, 16) || !aligned(w_v, 16) || !aligned(out, 16) ||
      !aligned(workspace, 256))
    return JF_ERR_INVALID_ARG;
  // a head at a time at least
  if (workspace_bytes < jf_latent_prefill_workspace_bytes(q_start, chunk_len, 1, 0))
    return JF_ERR_WORKSPACE_TOO_SMALL;
  LatentPrefill a;
  a.pool = latent_pool(*pool);
  a.pt = page_table_row;
  a.q = static_cast<const uint16_t*>(q);
  a.w_k = static_cast<const uint16_t*>(w_k);
  a.w_v = static_cast<const uint16_t*>(w_v);
  a.out = static_cast<uint16_t*>(out);
  a.q_start = q_start;
  a.C = chunk_len;
  a.H = num_heads;
  a.causal = causal;
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  a.status = static_cast<int32_t*>(workspace);
  return launch_latent_prefill(a, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

// ---------------------------------------------------------------------------
// Decode without a caller-supplied workspace: scratch in a file-scope device
// array.  In host code `jf_static_decode_ws` only names the symbol; its device
// address comes from cudaGetSymbolAddress, looked up once per device.
// ---------------------------------------------------------------------------
}  // extern "C"

static __device__ __align__(256) unsigned char jf_static_decode_ws[JF_STATIC_WORKSPACE_BYTES];

namespace {
constexpr int kMaxDevices = 256;
std::mutex g_static_ws_mu;
void* g_static_ws_ptr[kMaxDevices] = {};

// Device address of the static workspace on the current device (set-up on the
// first call per device, with that device current).
int static_workspace(void** out) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return JF_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return JF_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_static_ws_mu);
  if (!g_static_ws_ptr[dev]) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, jf_static_decode_ws) != cudaSuccess || !p) return JF_ERR_CUDA;
    g_static_ws_ptr[dev] = p;
  }
  *out = g_static_ws_ptr[dev];
  return JF_OK;
}
}  // namespace

extern "C" {

int jf_paged_decode_attn_noalloc(const jf_kv_pool* pool, const int32_t* page_table,
                                 int32_t pt_stride, const int32_t* context_lens, int32_t batch,
                                 const void* q, int32_t num_q_heads, float softmax_scale,
                                 void* out, int32_t num_splits, int32_t* err_flag, void* stream) {
  int st = check_pool(pool);
  if (st) return st;
  if (!page_table || !context_lens || !q || !out) return JF_ERR_INVALID_ARG;
  if (batch < 1 || batch > 65535 || pt_stride < 1 || num_q_heads < 1) return JF_ERR_INVALID_ARG;
  if (num_q_heads % pool->num_kv_heads) return JF_ERR_INVALID_ARG;
  if (num_q_heads / pool->num_kv_heads > 8) return JF_ERR_UNSUPPORTED;
  if (num_splits < 1 || num_splits > 65535) return JF_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return JF_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16)) return JF_ERR_INVALID_ARG;
  const size_t need = jf_attn_workspace_bytes(batch, num_q_heads, pool->num_kv_heads,
                                              pool->head_dim, num_splits);
  if (need == 0) return JF_ERR_INVALID_ARG;
  if (need > JF_STATIC_WORKSPACE_BYTES) return JF_ERR_WORKSPACE_TOO_SMALL;
  void* ws = nullptr;
  st = static_workspace(&ws);
  if (st) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // the status word is the only scratch that must start at zero
  if (cudaMemsetAsync(ws, 0, sizeof(int32_t), s) != cudaSuccess) return JF_ERR_CUDA;
  const Geom g = make_geom(*pool);
  CUtensorMap tmap;
  st = make_codes_map(g, pool->base, decode_box_rows(), &tmap);
  if (st) return st;
  st = launch_decode(g, *pool, tmap, page_table, pt_stride, context_lens, batch, q, num_q_heads,
                     softmax_scale, out, ws, num_splits, s);
  if (st) return st;
  if (err_flag &&
      cudaMemcpyAsync(err_flag, ws, sizeof(int32_t), cudaMemcpyDeviceToDevice, s) != cudaSuccess)
    return JF_ERR_CUDA;
  return JF_OK;
}

const char* jf_status_string(int status) {
  switch (status) {
    case JF_OK: return "JF_OK";
    case JF_ERR_INVALID_ARG: return "JF_ERR_INVALID_ARG";
    case JF_ERR_UNSUPPORTED: return "JF_ERR_UNSUPPORTED";
    case JF_ERR_WORKSPACE_TOO_SMALL: return "JF_ERR_WORKSPACE_TOO_SMALL";
    case JF_ERR_CUDA: return "JF_ERR_CUDA";
    default: return "JF_ERR_UNKNOWN";
  }
}

const char* jf_version(void) { return "jfkv 0.1 (sm_103a)"; }

}  // extern "C"
