// The latent cache format (JF_FMT_LATENT16) and what its kernels share.
//
// A position is one row of R + 64 bf16 values: the latent vector that the keys
// and values of all heads come from, and the rotated key channels that all heads
// share.  A page is page_size rows, so the pool is one array of num_pages x
// page_size rows.
#pragma once
#include "common.cuh"

namespace jfkv {

constexpr int LAT_ROT = 64;          // rotated key channels
constexpr int LAT_MAX_GROUPS = JF_LATENT_MAX_GROUPS;
constexpr int LAT_HEAD = 128;        // expanded form: a head's unrotated key and its value channels

struct LatentPool {
  const uint16_t* base;
  int64_t num_pages;
  int32_t P, log2P;
  int32_t R;            // latent channels
  int32_t row;          // R + 64
};

inline LatentPool latent_pool(const jf_kv_pool& p) {
  return LatentPool{static_cast<const uint16_t*>(p.base), p.num_pages, p.page_size,
                    __builtin_ctz((unsigned)p.page_size), p.head_dim - LAT_ROT, p.head_dim};
}

// One decode call: groups' shared runs (num_groups may be 0), and each request's own.
struct LatentDecode {
  LatentPool pool;
  const int32_t* prefix_table;     // [num_groups, prefix_stride]
  const int32_t* prefix_lens;      // [num_groups]
  int32_t prefix_stride, num_groups;
  const int32_t* page_table;       // [batch, pt_stride]
  const int32_t* context_lens;     // [batch]
  int32_t pt_stride, batch, H;
  const uint16_t* q;               // [batch, H, R + 64]
  uint16_t* out;                   // [batch, H, R]
  float scale_log2;                // softmax scale times log2(e)
  int32_t* status;
  int32_t first[LAT_MAX_GROUPS + 1];   // groups' first requests, and the batch
};

struct LatentPrefill {
  LatentPool pool;
  const int32_t* pt;               // the request's page-table row
  const uint16_t* q;               // [C, H, 192]
  const uint16_t* w_k;             // [H, 128, R]
  const uint16_t* w_v;             // [H, 128, R]
  uint16_t* out;                   // [C, H, 128]
  int32_t q_start, C, H, causal;
  float scale_log2;
  int32_t* status;
};

size_t latent_decode_workspace_bytes(int64_t batch, int64_t H, int64_t R, int64_t groups, int64_t sms);
size_t latent_prefill_workspace_bytes(int64_t q_start, int64_t C, int64_t H, int64_t sms);
int launch_latent_rows(const LatentPool& pool, const int32_t* page_table, int32_t pt_stride,
                       int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                       void* latent, int64_t latent_stride, void* k_rot, int64_t rot_stride,
                       int32_t n_rows, int32_t* err, bool read, cudaStream_t stream);
int launch_latent_decode(const LatentDecode& a, void* workspace, cudaStream_t stream);
int launch_latent_prefill(const LatentPrefill& a, void* workspace, size_t workspace_bytes, cudaStream_t stream);

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace jfkv
