// What the prefill kernels share: the per-launch argument block with its
// request table, and packed fp32 arithmetic.
#pragma once
#include "tc.cuh"

namespace jfkv {

constexpr int PF_BM = 128;   // MMA rows per CTA (256 per CTA pair)
constexpr int PF_BN = 64;    // positions per K/V tile
constexpr int PF_SM_WARPS = 4;   // one per TMEM lane quarter, one row per thread
constexpr int PF_KVBUF = 4;     // P V completion barriers, by tile index mod 4
constexpr float PF_TAU = 8.f;   // log2 headroom before the running max moves

// One request's chunk in a launch: its query tiles are CTAs tile0 ..
// tile0 + n_tiles2 - 1 (n_tiles2 even, so a CTA pair never spans requests).
struct PfReq {
  const int32_t* pt;    // its page-table row
  const uint16_t* q;    // its chunk's queries [C, Hq, D]
  uint16_t* out;        // [C, Hq, D]
  int32_t q_start, C, tile0, n_tiles2;
  int32_t row0;         // its first query's row in the launch (split partials)
};

constexpr int PF_MAX_REQ = 64;   // requests per launch

struct PrefillArgs {
  const uint8_t* pool;
  int64_t num_pages;
  int64_t page_bytes;
  int64_t codes_region;
  int64_t sb_base;
  int64_t sb_region;
  int32_t P, Hkv, Hq, G, QPC;
  int32_t causal;
  float scale_log2;
  int32_t* status;
  int32_t num_splits;   // > 1: history ranges per query tile, partials + merge
  float* part_ml;       // [rows * Hq][num_splits][2] (m, l)
  float* part_o;        // [rows * Hq][num_splits][D], unnormalized
  const float* qrot;     // TQ4: rotated queries H S_K q / sqrt(D), fp32 [rows * Hq][D]
  float cent[16];        // TQ4: centroids
  int32_t nreq;
  PfReq req[PF_MAX_REQ];
};

// Wave balance of one chunk over an 8-bit pool (kv8_prefill.cu).  CTA pairs run
// num_sms / 2 at a time; the pairs that fill whole waves run as they are, and the
// histories of the `tail` pairs left over, laid end to end, are cut into one piece
// per place, so that the last wave ends everywhere at once.  seg: the pieces' parts
// that belong to one pair, longest first (a place that gets a short part is free
// early and takes the rest of another).
constexpr int P8_MAX_SEG = 192;
struct P8Seg {
  uint16_t pair;        // in launch order
  uint8_t z, last;      // its partial row; whether the pair's later ones are unused
  uint16_t f0, f1;      // history range, in units of 1 / 32768 of the pair's tiles
};
struct P8Plan {
  int32_t whole;        // pairs run whole
  int32_t n;            // parts of the others (0: no plan)
  int32_t rows;         // queries of the others: the first of the chunk
  int32_t k;            // partial rows per query and head
  P8Seg seg[P8_MAX_SEG];
};
void kv8_prefill_plan(int64_t G, int64_t Hkv, int64_t q_start, int64_t chunk_len, bool causal,
                      int64_t num_sms, P8Plan* plan);

// One launch over an 8-bit pool (kv8_prefill.cu): ctas CTAs, splits history ranges,
// or those of a plan.
int launch_kv8_prefill(const Geom& g, const jf_kv_pool& pool, const PrefillArgs& a,
                       const P8Plan* plan, unsigned ctas, unsigned splits, cudaStream_t stream);

// packed fp32 pairs (Blackwell f32x2 arithmetic)
__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;\n" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t sub_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("sub.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

}  // namespace jfkv
