// Helpers of the latent cache's tensor-core kernels: pair MMAs on bf16, tiled copies, and
// the division of a launch's work into one run of equal length per CTA pair.
#pragma once
#include "latent.cuh"
#include "prefill.cuh"

namespace jfkv {

int bf16_rows_map(const void* base, int64_t channels, int64_t rows, int box_rows, CUtensorMap* map);
int bf16_chunks_map(const void* base, int64_t channels, int64_t rows, int box_chunks, CUtensorMap* map);
int sm_count();

inline int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, int b_mn) {
  return tc::idesc_f16_f32(M, N, 0, b_mn) | (1u << 7) | (1u << 10);
}

// Pair MMA, both operands in shared memory, issued where `leader` is set by a warp that runs the
// issuing code as a whole: control flow and operands are then uniform values.  (Run by one thread
// alone, each descriptor was moved to uniform registers first: 72 to 100 cycles an instruction for
// the 32 to 64 that the product takes.)
__device__ __forceinline__ void mma2_ss_if(uint32_t leader, uint32_t d, uint64_t a, uint64_t b,
                                           uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}

// whether the phase is over, without waiting
__device__ __forceinline__ bool mbar_test(uint64_t* bar, int phase) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}\n"
      : "=r"(ok) : "r"(smem_u32(bar)), "r"((uint32_t)(phase & 1)) : "memory");
  return ok != 0;
}

__device__ __forceinline__ uint32_t elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
               : "=r"(p));
  return p;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];\n"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];\n"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}

// 32 lanes x 16 columns of 32-bit words
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15,%16};\n"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
        "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]),
        "r"(v[15])
      : "memory");
}

// 16 lanes x 32 columns of 32-bit words in 16 x 8 pieces: of piece i thread t has columns 8 i + 2 (t % 4)
// and the next of lane t / 4 in v[4 i], v[4 i + 1], of lane t / 4 + 8 in v[4 i + 2], v[4 i + 3]
__device__ __forceinline__ void ld16_32(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15},"
      " [%16];\n"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]),
        "=r"(v[15])
      : "r"(taddr));
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n"
               ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// The block's end, all threads together; whether no wait gave up.  Where one did, copies and products may still
// be under way: they get a millisecond, a thousand times what they take, before the memory is released.
__device__ __forceinline__ bool settle(bool ok) {
  if (!__syncthreads_or(!ok)) return true;
  for (int i = 0; i < 100; ++i) __nanosleep(10000);
  return false;
}

// Both CTAs of the pair are here.  Relaxed: nothing is handed over, and a release would first wait for
// this CTA's stores to reach memory, which the kernel's end does anyway.  Only where every arrival at either
// CTA's barriers has been waited for there, those of the products' commits among them: nothing orders one
// still on its way, not the one of a later commit.
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.aligned;\n" ::: "memory");
}

// brings memory into the L2 cache, 16-byte aligned
__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(p), "r"(bytes) : "memory");
}

// x / y, in 32 bits where both have no more
__device__ __forceinline__ uint64_t divide(uint64_t x, uint64_t y) {
  return (x | y) >> 32 ? x / y : (uint64_t)((uint32_t)x / (uint32_t)y);
}
// 2^32 / pairs, rounded up
inline uint32_t pairs_inverse(int64_t pairs) {
  const uint64_t x = (((uint64_t)1 << 32) + pairs - 1) / pairs;
  return x >> 32 ? 0xFFFFFFFFu : (uint32_t)x;
}
struct PairRuns {   // floor(units * p / pairs); inv is pairs_inverse(pairs)
  int64_t units, each;
  uint32_t rest, pairs, inv;
  __device__ __forceinline__ PairRuns(int64_t u, int n, uint32_t v) : units(u), pairs((uint32_t)n), inv(v) {
    int64_t left;
    if ((uint64_t)u >> 32) {
      each = (int64_t)((uint64_t)u / pairs);
      left = u - each * n;
    } else {   // the product with the inverse is off by one at most
      each = __umulhi((uint32_t)u, inv);
      left = u - each * n;
      if (left < 0) {
        --each;
        left += n;
      }
      if (left >= n) {
        ++each;
        left -= n;
      }
    }
    rest = (uint32_t)left;
  }
  __device__ __forceinline__ int64_t first(int p) const {
    return each * p + __umulhi((uint32_t)p * rest, inv);   // p * rest below 2^14: exact
  }
  // the pair that has unit u: the last p with first(p) <= u
  __device__ __forceinline__ int of(int64_t u) const {
    return (int)divide((uint64_t)(u + 1) * pairs + (uint64_t)units - 1, (uint64_t)units) - 1;
  }
};

// the page of the 64 positions from pos, as a row of the pool; past the map's end (the copy then
// brings zeros) where there is none
__device__ __forceinline__ int half_row(const LatentPool& p, const int32_t* pt, int pos, int len,
                                        int32_t* status) {
  const int end = (int)(p.num_pages << p.log2P);
  if (pos >= len) return end;
  const int32_t page = __ldg(pt + (pos >> p.log2P));
  if (page < 0 || page >= p.num_pages) {
    if (status) flag_error(status, JF_DEV_ERR_PAGE_ID);
    return end;
  }
  return (page << p.log2P) + (pos & (p.P - 1));
}

}  // namespace jfkv
