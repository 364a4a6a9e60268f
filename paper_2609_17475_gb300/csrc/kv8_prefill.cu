// Prefill-chunk attention over the 8-bit block-scaled cache on the 5th-generation
// tensor cores.
//
// The tiling is prefill.cu's: a CTA holds 128 (query, head) rows of one KV head,
// two CTAs form a pair whose M = 256 MMAs share every 64-position K/V tile, S is
// taken over pairs of tiles (N = 128) into two TMEM buffers, P (fp16) replaces
// S columns already read, O stays in TMEM.  What the 8-bit codes change:
//  * S = Q K^T multiplies the codes as they lie in the pool (kind::f8f6f4): TMA
//    brings K rows straight into the MMA's swizzled layout and nothing is
//    dequantized.  Q, which needs more than e4m3's 4 bits, enters as a sum of two
//    terms, hi in e4m3 and lo in e5m2, of the row scaled so that its largest element
//    lies in [2^7, 2^8).  From 2^-6 up hi is off by at most 8 units of bf16's last
//    place, a whole number that e5m2's 3 bits hold: elements within 2^13 of the largest
//    enter exactly.  Below, hi is off by at most 2^-10 and lo's rounding of that by
//    2^-14, 2^-21 of the largest.  (With lo in e4m3, whose least step is 2^-9, the
//    bounds were 2^9 and 2^-17.)  Two 8-bit products take the time of one 16-bit product.
//  * P V stays fp16 -- P has to keep small weights, which e4m3 cannot -- with V's
//    codes widened to fp16 (exact) by four warps.
//  * The block scales are powers of two and a half tile is a block: K's multiplies
//    the fp32 score, V's exponent is added to it, so that P carries it, and l
//    takes it out again (kv8_decode.cu has the identity).
//  * With half of the dequantization gone, eight warps do the softmax: two groups
//    of four take the even and the odd tiles, so that a pair's two tiles are
//    worked on side by side while the tensor core runs the next pair's S and the
//    last pair's P V.  A row's reference maximum moves only when a score exceeds
//    it by 2^14; the groups agree on it tile by tile through shared memory, but
//    only after a tile's exponentials, which are worked out with the last known
//    reference and again where it turns out to have moved.
// Warp roles (each CTA):
//   warp 0       TMEM; CTA 0's lane 0 issues every MMA of the pair, CTA 1's lane 0
//                passes its K arrivals on to CTA 0
//   warp 1       lane 0 loads this CTA's K halves (32 positions of each tile) by
//                TMA into three pair buffers, and the 128 bytes of each V row that
//                hold its half into four staging tiles
//   warps 2-5    V halves (D/2 columns of each tile) -> fp16, four tile buffers (six at
//                D = 128)
//   warps 6-13   Q at the start; softmax; O / l -> bf16 (or the split's partial)
// Bound: the tensor core, at the clock its power allows.  1,596 queries after 30,720
// positions (24 / 4 heads x 256, two full waves) 738 us, 1,670 TFLOP/s: 0.88 of the
// bf16 burst rate, 0.97 of the sustained one.  At D = 128 a tile has half the products for
// the same exponentials, and the softmax warps set the pace: 798 queries so, one wave,
// 294 us, 1,040 TFLOP/s.  77 queries after 4,001 positions (8 / 2 heads x 128), history split 8
// ways: 19.5 us of launches, Q's way in, eight tiles one after the other and the merge.
// Waits acquire at CTA scope: what a barrier publishes is read by the tensor core,
// from TMEM behind a tcgen05 fence, or from this CTA's own shared memory, never by
// plain loads from the other CTA's (cluster scope cost 4 % at D = 256, 8 % at 128).
#include <cmath>

#include "kv8.cuh"
#include "prefill.cuh"

namespace jfkv {

int kv8_tensor_map(const Geom& g, void* base, int halves, int rows, int kv, CUtensorMap* map);

constexpr int P8_KBUF = 3;                 // K pair buffers
constexpr int P8_SBUF = 4;                 // V staging tiles
constexpr int P8_V_WARP0 = 2, P8_SM_WARP0 = 6;
constexpr int P8_THREADS = 32 * 14;
constexpr float P8_TOP = 14.f;             // P stays below 2^14
constexpr float P8_SET = 6.f;              // a new reference puts the largest P at 2^6

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Where a CTA's results go, kept in shared memory with the rows' places so that the
// softmax loop holds none of it in registers (1,596 queries after 30,720 positions,
// when it was moved: 774 -> 760 us).
struct P8Out {
  uint8_t* to;          // the output, or the partials O
  int32_t split;
  int32_t unused;       // partial rows after this one that no part of the plan writes
};

template <int D>
struct P8Smem {
  static constexpr int NB = D / 128;                     // 128-byte blocks of a row
  static constexpr int Q_BYTES = PF_BM * D;              // one term: [D/128][128 rows][128 B]
  static constexpr int KP_BYTES = PF_BN * D;             // [D/128][64 rows][128 B]
  static constexpr int VT_BYTES = PF_BN * (D / 2) * 2;   // [D/128][64 rows][128 B]
  static constexpr int OFF_Q = 0;                        // hi, then lo
  static constexpr int OFF_K = 2 * Q_BYTES;
  static constexpr int OFF_V = OFF_K + P8_KBUF * KP_BYTES;
  static constexpr int VS_BYTES = PF_BN * 128;           // staged codes: [64 rows][128 B]
  static constexpr int NSB = (512 - D) / (2 * PF_BN);    // S/P buffers: what O leaves of TMEM
  static constexpr int VBUF = 2 * NSB;                   // V tile buffers
  static constexpr int OFF_S = OFF_V + VBUF * VT_BYTES;
  static constexpr int OFF_BAR = OFF_S + P8_SBUF * VS_BYTES;
  static constexpr int OFF_M = OFF_BAR + 512;            // [128] reference maxima
  static constexpr int OFF_L = OFF_M + PF_BM * 4;        // [2 groups][128] (m, l)
  static constexpr int OFF_X = OFF_L + 2 * PF_BM * 8;    // [128] largest magnitude of a Q row
  static constexpr int OFF_R = OFF_X + PF_BM * 4;        // [128] output row, -1: none
  static constexpr int OFF_OUT = OFF_R + PF_BM * 8;      // P8Out
  static constexpr int OFF_NAN = OFF_OUT + 16;           // [D + 1] first positions of NaN (below)
  static constexpr int OFF_LIM = OFF_NAN + (D + 4) * 4;  // [128] last position a row sees
  static constexpr int TOTAL = 1024 + OFF_LIM + PF_BM * 4;
  // at the end O's rows pass through what held Q, K and V on their way out
  static_assert(PF_BM * D * 4 <= OFF_BAR, "O rows");
  static_assert(TOTAL <= 227 * 1024, "shared memory per CTA");
};

// exponent of a Q row whose largest magnitude has the bf16 bits mx: mx 2^-e in [2^7, 2^8)
__device__ __forceinline__ int q_exp(uint32_t mx) {
  return mx >= 0x80u ? max((int)(mx >> 7) - 127 - 7, -100) : -100;
}

__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t x, uint32_t y, uint32_t z,
                                             uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n"
               ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

__device__ __forceinline__ uint32_t e5m2x4_of_f16x2(uint32_t lo, uint32_t hi) {
  uint32_t r;
  asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e5m2x2.f16x2 a, %1;\n"
      "cvt.rn.satfinite.e5m2x2.f16x2 b, %2;\nmov.b32 %0, {a, b};\n}\n"
      : "=r"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// largest x of the LPR lanes that hold a row
template <int LPR>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  if constexpr (LPR == 32) {
    return __reduce_max_sync(0xffffffffu, x);
  } else {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
  }
}

// A value that is NaN and that some query of the pair does not see would reach that query as
// 0 * NaN.  It enters the product as zero instead, and the first such position of its channel
// is kept in both CTAs (`first`, shared; element D is the first of all channels), so that the
// outputs of the queries that do see it can be made NaN at the end.  (798 queries at
// D = 128 290 -> 294 us; at D = 256 no difference.)
template <int D>
__device__ __noinline__ void note_nan(uint32_t mask, int d, int pos, uint32_t first) {
  for (uint32_t rank = 0; rank < 2; ++rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(first), "r"(rank));
    for (int i = 0; i < 5; ++i)
      if (i == 4 || ((mask >> (8 * i)) & 1u))
        asm volatile("red.relaxed.cluster.shared::cluster.min.s32 [%0], %1;\n"
                     ::"r"(at + 4 * (i == 4 ? D : d + i)), "r"(pos) : "memory");
  }
}
// the codes of channels d .. d + 3 with NaN replaced by zero
template <int D>
__device__ __forceinline__ uint32_t without_nan(uint32_t w, int d, int pos, uint32_t first) {
  const uint32_t mask = __vcmpeq4(w & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
  if (mask) note_nan<D>(mask, d, pos, first);
  return w & ~mask;
}

struct P8NoPlan {};
template <bool PLAN> struct P8PlanArg { using type = P8Plan; };
template <> struct P8PlanArg<false> { using type = P8NoPlan; };

// PLAN: whole pairs, then the plan's parts; otherwise gridDim.z ranges of every pair.
template <int D, bool PLAN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P8_THREADS, 1)
kv8_prefill_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ PrefillArgs a,
                   const __grid_constant__ typename P8PlanArg<PLAN>::type plan) {
  using L = P8Smem<D>;
  constexpr uint32_t IDHI = tc::idesc_e4m3_f32(2 * PF_BM, 2 * PF_BN);   // a tile pair
  constexpr uint32_t IDLO = IDHI | (1u << 7);                           // A's type: e5m2
  constexpr uint32_t IDPV = tc::idesc_f16_f32(2 * PF_BM, D, 0, 1);
  // S of pair i is issued before P V of pair i - AHEAD, so that the softmax of a pair may
  // run while the P V of AHEAD pairs before it are outstanding: V buffers and barriers for
  // the tiles of NSB pairs, or an arrival (pv_ready) or a wait (pv_done) would meet the
  // phase before its own.  798 queries at D = 128, three S/P buffers for two: 304 -> 296 us.
  constexpr int NSB = L::NSB, AHEAD = NSB - 1, PVR = L::VBUF;
  static_assert(PVR <= 6, "barriers");

  extern __shared__ uint8_t smraw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smraw) + 1023) &
                                           ~static_cast<uintptr_t>(1023));
  uint8_t* const sQ = sm + L::OFF_Q;
  uint8_t* const sK = sm + L::OFF_K;
  uint8_t* const sV = sm + L::OFF_V;
  uint8_t* const sS = sm + L::OFF_S;
  float* const s_m = reinterpret_cast<float*>(sm + L::OFF_M);
  float2* const s_ml = reinterpret_cast<float2*>(sm + L::OFF_L);
  int64_t* const s_row = reinterpret_cast<int64_t*>(sm + L::OFF_R);
  P8Out* const s_out = reinterpret_cast<P8Out*>(sm + L::OFF_OUT);
  uint32_t* const s_x = reinterpret_cast<uint32_t*>(sm + L::OFF_X);
  int32_t* const s_nan = reinterpret_cast<int32_t*>(sm + L::OFF_NAN);
  int32_t* const s_lim = reinterpret_cast<int32_t*>(sm + L::OFF_LIM);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sm + L::OFF_BAR);
  // On CTA 0, where the pair's MMAs are issued:
  uint64_t* const k_full = bars + 0;     // [3] both CTAs' K halves of a pair have landed
  uint64_t* const pv_ready = bars + 3;   // [PVR] both CTAs' V halves and P of tile j % PVR stored
  // on each CTA:
  uint64_t* const k_land = bars + 9;     // [3] CTA 1: its K halves have landed
  uint64_t* const s_full = bars + 12;    // [3] S of pair i % 3 done (its K buffer is free)
  uint64_t* const pv_done = bars + 15;   // [PVR] P V of tile j % PVR done
  uint64_t* const m_bar = bars + 21;     // [2 groups][4 quarters] the group's reference is set
  uint64_t* const s_land = bars + 29;    // [4] staged V codes have landed
  uint64_t* const s_free = bars + 33;    // [4] and been read by the 4 V warps
  uint64_t* const q_ready = bars + 37;   // on CTA 0: both CTAs' Q rows stored
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 38);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);   // uniform
  const int lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  // CTA pairs in launch order, as in prefill.cu: the KV heads of a pair of query
  // tiles are consecutive, latest (longest) tiles first
  int pair = (int)(blockIdx.x >> 1), z = (int)blockIdx.z;
  bool split = a.num_splits > 1;
  int f0 = 0, f1 = 0, last = 0;
  if constexpr (PLAN) {
    split = pair >= plan.whole;
    if (split) {
      const P8Seg& sg = plan.seg[pair - plan.whole];
      pair = sg.pair;
      z = sg.z;
      f0 = sg.f0;
      f1 = sg.f1;
      last = sg.last;
    }
  }
  const int kvh = pair % a.Hkv;
  const int tile = (pair / a.Hkv) * 2 + (int)(blockIdx.x & 1);
  int ri = 0;
  for (int i = 1; i < a.nreq; ++i)
    if (tile >= a.req[i].tile0) ri = i;
  const PfReq& rq = a.req[ri];
  const int32_t* const pt = rq.pt;
  const int q_start = rq.q_start, C = rq.C;
  const int bx = tile - rq.tile0;
  const int qt = rq.n_tiles2 - 1 - bx;
  const int qt_partner = rq.n_tiles2 - 1 - (bx ^ 1);
  const int q0 = qt * a.QPC;
  const int nq = max(0, min(a.QPC, C - q0));
  const int rows = nq * a.G;
  const int total = q_start + C;
  auto kmax_of = [&](int t) {   // positions a query tile attends (0 for a padding tile)
    const int first = t * a.QPC;
    const int n = max(0, min(a.QPC, C - first));
    return n == 0 ? 0 : (a.causal ? q_start + first + n : total);
  };
  const int kmax_pair = max(kmax_of(qt), kmax_of(qt_partner));
  const int ntiles_all = (kmax_pair + PF_BN - 1) / PF_BN;
  int jb = 0, je = ntiles_all;
  if (PLAN && split) {
    jb = (int)(((int64_t)ntiles_all * f0) >> 15);
    je = (int)(((int64_t)ntiles_all * f1) >> 15);
  } else if (split) {
    jb = (int)(((int64_t)ntiles_all * z) / a.num_splits);
    je = (int)(((int64_t)ntiles_all * (z + 1)) / a.num_splits);
  }
  const int ntiles = je - jb;
  const int npairs = (ntiles + 1) >> 1;

  const int quarter = warp & 3;                // TMEM lanes a softmax warp may access
  const int group = warp >= P8_SM_WARP0 + 4 ? 1 : 0;
  const int r = quarter * 32 + lane;
  const bool row_ok = r < rows;
  const int qi = row_ok ? r / a.G : 0;
  if (warp >= P8_SM_WARP0 && group == 0) {
    const int64_t at = (int64_t)(q0 + qi) * a.Hq + kvh * a.G + r % a.G;
    s_row[r] = !row_ok ? -1 : split ? ((int64_t)rq.row0 * a.Hq + at) * a.num_splits + z : at;
    s_lim[r] = q_start + q0 + qi;
  }
  if (threadIdx.x == 0)
    *s_out = P8Out{split ? reinterpret_cast<uint8_t*>(a.part_o) : reinterpret_cast<uint8_t*>(rq.out),
                   split ? 1 : 0, last ? a.num_splits - 1 - z : 0};
  const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
  for (int i = threadIdx.x; i <= D; i += P8_THREADS) s_nan[i] = 0x7FFFFFFF;
  if (threadIdx.x == 0) {
    prefetch_tensormap(&kmap);
    mbar_init(q_ready, 2 * 2 * PF_SM_WARPS);
    for (int i = 0; i < PVR; ++i) {
      mbar_init(&pv_ready[i], 2 * (4 + PF_SM_WARPS));   // 4 V and 4 softmax warps of each CTA
      mbar_init(&pv_done[i], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&m_bar[i], 1);
      mbar_init(&m_bar[4 + i], 1);
      mbar_init(&s_land[i], 1);
      mbar_init(&s_free[i], 4);
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(&k_full[i], 2);   // CTA 0's own copies, CTA 1's arrival
      mbar_init(&k_land[i], 1);
      mbar_init(&s_full[i], 1);
    }
    fence_barrier_init();
  }
  if (warp == 0) tc::alloc2(tmem_slot, 512);
  asm volatile("griddepcontrol.wait;\n" ::: "memory");   // what came before has been written
  // 16 Q rows to a softmax warp, a whole row (two at D = 128) per load, under way while
  // the CTAs meet
  constexpr int LPR = D / 8;                   // lanes of a row, 8 elements each
  constexpr int RPI = 32 / LPR, NI = 16 / RPI;
  const int qpiece = lane % LPR;
  const int qr0 = (warp - P8_SM_WARP0) * 16 + lane / LPR;
  uint4 qv[NI];
  if (warp >= P8_SM_WARP0) {
    const uint32_t inv = (65535u + a.G) / (uint32_t)a.G;   // row / G = row * inv >> 16 below 128
    const uint16_t* const src = rq.q + ((int64_t)q0 * a.Hq + kvh * a.G) * D + qpiece * 8;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = qr0 + i * RPI;
      const int at = (int)((uint32_t)row * inv >> 16);
      qv[i] = make_uint4(0u, 0u, 0u, 0u);
      if (row < rows)
        qv[i] = *reinterpret_cast<const uint4*>(src + ((int64_t)at * a.Hq + (row - at * a.G)) * D);
    }
  }
  tc::fence_before();
  __syncthreads();
  tc::cluster_sync();   // both CTAs: barriers initialized, TMEM allocated
  tc::fence_after();
  // All 512 columns are this CTA's, so they start at 0; addresses known to the compiler
  // are worth it where MMAs are issued (1,596 queries after 30,720 positions 758 us with
  // the address from the slot, 725 so; 798 at D = 128 327 and 304).
  constexpr uint32_t tbase = 0;
  const uint32_t tO = tbase;
  const uint32_t tS = tbase + D;

  const int log2P = 31 - __clz(a.P);           // P is a power of two
  auto page_of = [&](int j) -> int {           // of tile j (P >= 64: a tile lies in one page)
    return j < ntiles ? __ldg(pt + (((jb + j) * PF_BN) >> log2P)) : -1;
  };

  // ---- softmax warps: Q rows as two 8-bit terms (K-major, 128-byte swizzle: 16-byte
  // piece m of row r at block m / 8, piece (m % 8) ^ (r % 8)) -------------------------
  float smul = 0.f;                            // score = smul * S
  if (warp >= P8_SM_WARP0) {
    const bool zero = a.scale_log2 == 0.f;     // zero scores
    uint8_t* const at = sQ + (qpiece >> 4) * (PF_BM * 128) + (qpiece & 1) * 8;
    const int m7 = (qpiece >> 1) & 7;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = qr0 + i * RPI;
      const uint32_t ws[4] = {qv[i].x, qv[i].y, qv[i].z, qv[i].w};
      uint32_t m2 = 0;                         // largest magnitudes
#pragma unroll
      for (int k = 0; k < 4; ++k) m2 = __vmaxu2(m2, ws[k] & 0x7FFF7FFFu);   // bits in order
      const uint32_t mx = row_max<LPR>(max(m2 & 0xFFFFu, m2 >> 16));
      if (qpiece == 0) s_x[row] = mx;
      float qs = two8(-q_exp(mx));
      if (a.scale_log2 < 0.f) qs = -qs;        // the scale's sign goes to Q
      uint32_t hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
      if (!zero) {
        // by way of fp16, which holds what e5m2 does not round to 0 (2^-17) exactly
        uint32_t f[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          f[k] = pack_f16x2(bf16lo_to_f32(ws[k]) * qs, bf16hi_to_f32(ws[k]) * qs);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          hi[k] = e4m3x4_of_f16x2(f[2 * k], f[2 * k + 1]);
          uint32_t h0, h1;
          f16x4_of_e4m3(hi[k], h0, h1);
          lo[k] = e5m2x4_of_f16x2(sub_f16x2(f[2 * k], h0), sub_f16x2(f[2 * k + 1], h1));
        }
      }
      uint8_t* const to = at + row * 128 + ((m7 ^ (row & 7)) << 4);
      *reinterpret_cast<uint2*>(to) = make_uint2(hi[0], hi[1]);
      *reinterpret_cast<uint2*>(to + L::Q_BYTES) = make_uint2(lo[0], lo[1]);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) tc::arrive_cluster(q_ready, 0);
    asm volatile("bar.sync 1, %0;\n" ::"n"(2 * PF_SM_WARPS * 32) : "memory");   // s_x
    const uint32_t mx = s_x[r];
    smul = fabsf(a.scale_log2) * two8(q_exp(mx));
    // the factor stays positive under a block's smallest scale, 2^-40: the -inf of positions
    // not seen, times zero, would be NaN.  2^-86 moves no score by more than 2^-20.
    if (smul < 0x1p-86f) smul = 0x1p-86f;
    // e4m3 has no infinity: a row that holds one, or a NaN, is NaN by its factor
    if (mx >= 0x7F80u) smul = __uint_as_float(0x7FC00000u);
  }

  float m_own = -INFINITY, l = 0.f;   // softmax: the reference at this group's last tile
  bool ok = true;
  if (warp == 0) {
    if (rank == 0) {
      // ================= MMA issuer =================
      // The whole warp runs this loop, so that its control flow and the operands'
      // descriptors are uniform values; lane 0 alone issues (the loop run by lane 0
      // alone moved every descriptor to uniform registers first, which took longer
      // than the products: 1,596 queries after 30,720 positions 982 us, 924 after).
      const uint64_t qd = tc::sdesc_sw128(smem_u32(sQ), 16, 1024);
      const uint64_t kd = tc::sdesc_sw128(smem_u32(sK), 16, 1024);
      const uint64_t vd = tc::sdesc_sw128(smem_u32(sV), PF_BN * 128, 1024);
      const uint32_t leader = lane == 0;
      auto wait = [&](uint64_t* bar, int phase) {
        return __all_sync(0xffffffffu, mbar_wait_bounded(bar, phase & 1)) != 0;
      };
      // S of pair i (column n = K row n of CTA 0 for n < 64, row n - 64 of CTA 1
      // otherwise: position 32 rank + n % 32 of tile 2i + (n % 64) / 32), then P V of
      // the tiles of pair i - AHEAD
      int jn = 0;   // next tile whose P V is due
      ok = wait(q_ready, 0);
      for (int i = 0; i < npairs + AHEAD && ok; ++i) {
        if (i < npairs) {
          const int kb = i % P8_KBUF;
          ok = wait(&k_full[kb], i / P8_KBUF);
          if (!ok) break;
          tc::fence_after();
          const uint64_t kd_i = kd + (uint64_t)(kb * (L::KP_BYTES >> 4));
          const uint32_t d = tS + (i % NSB) * (2 * PF_BN);
#pragma unroll
          for (int ks = 0; ks < 2 * (D / 32); ++ks) {   // hi's steps, then lo's
            const int k = ks % (D / 32);
            tc::mma2_ss_f8_if(leader, d,
                              qd + (((ks / (D / 32)) * L::Q_BYTES + (k >> 2) * (PF_BM * 128) +
                                     (k & 3) * 32) >> 4),
                              kd_i + (((k >> 2) * (PF_BN * 128) + (k & 3) * 32) >> 4),
                              ks < D / 32 ? IDHI : IDLO, ks ? 1u : 0u);
          }
          tc::commit2_both_if(leader, &s_full[kb]);
        }
        for (const int upto = min(2 * (i - AHEAD + 1), ntiles); jn < upto; ++jn) {
          const int vb = jn % PVR;
          ok = wait(&pv_ready[vb], jn / PVR);
          if (!ok) break;
          tc::fence_after();
          const uint64_t vd_j = vd + (uint64_t)(vb * (L::VT_BYTES >> 4));
          const uint32_t tp = tS + ((jn >> 1) % NSB) * (2 * PF_BN) + (jn & 1) * 32;
#pragma unroll
          for (int k = 0; k < PF_BN / 16; ++k)
            tc::mma2_ts_if(leader, tO, tp + 8 * k, vd_j + ((k * 2048) >> 4), IDPV,
                           (jn > 0 || k > 0) ? 1u : 0u);
          tc::commit2_both_if(leader, &pv_done[vb]);
        }
      }
    } else if (rank == 1 && lane == 0) {
      // ================= CTA 1's K arrivals =================
      for (int i = 0; i < npairs && ok; ++i) {
        const int kb = i % P8_KBUF;
        if (!mbar_wait_bounded(&k_land[kb], (i / P8_KBUF) & 1)) { ok = false; break; }
        tc::arrive_cluster(&k_full[kb], 0);
      }
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    __syncwarp();
  } else if (warp == 1) {
    // ================= K halves and V codes by TMA =================
    if (lane == 0) {
      int pg[2] = {page_of(0), page_of(1)};
      for (int i = 0; i < npairs && ok; ++i) {
        const int tiles = min(2, ntiles - 2 * i);
        int page[2] = {pg[0], pg[1]};
        pg[0] = page_of(2 * i + 2);   // a pair ahead
        pg[1] = page_of(2 * i + 3);
        for (int u = 0; u < tiles; ++u)
          if (page[u] < 0 || page[u] >= a.num_pages) {   // past the map's end: zeros
            flag_error(a.status, JF_DEV_ERR_PAGE_ID);
            page[u] = (int)min(a.num_pages, (int64_t)0x7FFFFFFF);
          }
        const int kb = i % P8_KBUF;
        uint64_t* const land = rank == 0 ? &k_full[kb] : &k_land[kb];
        if (i >= P8_KBUF && !mbar_wait_bounded(&s_full[kb], ((i / P8_KBUF) - 1) & 1)) {
          ok = false;
          break;
        }
        mbar_arrive_expect_tx(land, (uint32_t)tiles * L::NB * 4096);
        for (int u = 0; u < tiles; ++u) {
          const int row = kvh * a.P + (((jb + 2 * i + u) * PF_BN) & (a.P - 1));
          for (int b = 0; b < L::NB; ++b)
            tma_load_5d(sK + kb * L::KP_BYTES + b * (PF_BN * 128) + u * (32 * 128), &kmap, 0, b,
                        row + 32 * (int)rank, 0, page[u], land);
        }
        for (int u = 0; u < tiles; ++u) {
          const int j = 2 * i + u, sb = j % P8_SBUF;
          if (j >= P8_SBUF && !mbar_wait_bounded(&s_free[sb], ((j / P8_SBUF) - 1) & 1)) {
            ok = false;
            break;
          }
          mbar_arrive_expect_tx(&s_land[sb], L::VS_BYTES);
          const int row = kvh * a.P + (((jb + j) * PF_BN) & (a.P - 1));
          for (int h = 0; h < 2; ++h)
            tma_load_5d(sS + sb * L::VS_BYTES + h * (32 * 128), &kmap, 0, D == 256 ? (int)rank : 0,
                        row + 32 * h, 1, page[u], &s_land[sb]);
        }
      }
      if (!ok) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
    __syncwarp();
  } else if (warp < P8_SM_WARP0) {
    // ================= V halves -> fp16 =================
    // thread t: position t % 64, and of this CTA's D/2 columns the 64 (D = 256) or
    // 32 (D = 128) that t / 64 names
    const int e = (int)threadIdx.x - 32 * P8_V_WARP0;
    const int t = e % PF_BN, part = e / PF_BN;
    constexpr int NLD = D / 64;                      // 16-byte pieces of codes
    const int code0 = D == 256 ? 4 * part : 4 * (int)rank + 2 * part;
    const uint32_t src = smem_u32(sS) + t * 128;
    // its 16-byte pieces (8 fp16) in the tile [D/128][64 rows][128 B]
    uint8_t* const dst = sV + (D == 256 ? part : 0) * (PF_BN * 128) + t * 128;
    const int piece0 = D == 256 ? 0 : 4 * part;
    const int seen = a.causal ? q_start + min(qt, qt_partner) * a.QPC : 0x7FFFFFFF;   // by every row
    const int d0 = (D == 256 ? 128 * (int)rank : 0) + 16 * code0;                     // first channel
    for (int j = 0; j < ntiles; ++j) {
      const int sb = j % P8_SBUF, vb = j % PVR;
      if (!mbar_wait_bounded(&s_land[sb], (j / P8_SBUF) & 1)) { ok = false; break; }
      uint4 c[NLD];
#pragma unroll
      for (int u = 0; u < NLD; ++u)
        c[u] = ld_shared_v4(src + sb * L::VS_BYTES + (((code0 + u) ^ (t & 7)) << 4));
      const int pos = (jb + j) * PF_BN + t;
      if (pos >= kmax_pair) {   // a slot no query sees: whatever it holds
#pragma unroll
        for (int u = 0; u < NLD; ++u) c[u] = make_uint4(0u, 0u, 0u, 0u);
      } else if (pos > seen) {
#pragma unroll
        for (int u = 0; u < NLD; ++u) {
          const uint32_t first = smem_u32(s_nan);
          c[u].x = without_nan<D>(c[u].x, d0 + 16 * u, pos, first);
          c[u].y = without_nan<D>(c[u].y, d0 + 16 * u + 4, pos, first);
          c[u].z = without_nan<D>(c[u].z, d0 + 16 * u + 8, pos, first);
          c[u].w = without_nan<D>(c[u].w, d0 + 16 * u + 12, pos, first);
        }
      }
      uint32_t f[NLD][8];
#pragma unroll
      for (int u = 0; u < NLD; ++u) {
        f16x4_of_e4m3(c[u].x, f[u][0], f[u][1]);
        f16x4_of_e4m3(c[u].y, f[u][2], f[u][3]);
        f16x4_of_e4m3(c[u].z, f[u][4], f[u][5]);
        f16x4_of_e4m3(c[u].w, f[u][6], f[u][7]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_free[sb]);
      if (j >= PVR && !mbar_wait_bounded(&pv_done[vb], ((j / PVR) - 1) & 1)) {
        ok = false;
        break;
      }
#pragma unroll
      for (int u = 0; u < NLD; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<uint4*>(dst + vb * L::VT_BYTES +
                                    (((piece0 + 2 * u + h) ^ (t & 7)) << 4)) =
              make_uint4(f[u][4 * h], f[u][4 * h + 1], f[u][4 * h + 2], f[u][4 * h + 3]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::arrive_cluster(&pv_ready[vb], 0);
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
  } else {
    // ================= softmax: the tiles j = group, group + 2, ... =================
    // padding rows see every position: their Q rows are zero and their outputs
    // are not stored
    const int limit = (row_ok && a.causal) ? q_start + q0 + qi : kmax_pair - 1;
    // the two K and two V scales of a tile, loaded a tile of the group ahead (the
    // page id two)
    float2 ks, vs, ks_next = make_float2(1.f, 1.f), vs_next = ks_next;
    auto load_scales = [&](int j, int page) {
      ks_next = vs_next = make_float2(1.f, 1.f);
      if (page >= 0 && page < a.num_pages) {
        const uint8_t* p = a.pool + (int64_t)page * a.page_bytes + a.sb_base +
                           (kvh * (a.P / KV8_BLOCK) + (((jb + j) * PF_BN) & (a.P - 1)) / KV8_BLOCK) * 4;
        // written by an append that this grid may overlap: no read-only load
        ks_next = *reinterpret_cast<const float2*>(p);
        vs_next = *reinterpret_cast<const float2*>(p + a.sb_region);
      }
    };
    load_scales(group, page_of(group));
    int page_next = page_of(group + 2);
    for (int j = group; j < ntiles; j += 2) {
      ks = ks_next;
      vs = vs_next;
      load_scales(j + 2, page_next);
      page_next = page_of(j + 4);
      const int pi = j >> 1;
      const int ev0 = exp8_of_scale(vs.x), ev1 = exp8_of_scale(vs.y);
      const float k0 = smul * two8(exp8_of_scale(ks.x)), k1 = smul * two8(exp8_of_scale(ks.y));
      const int key0 = (jb + j) * PF_BN;
      // tile j's S: positions 0..31 in columns 32 (j & 1) .., 32..63 in columns
      // 64 + 32 (j & 1) .. of its pair's buffer; P_j goes to columns 32 (j & 1) ..
      const uint32_t tb = tS + (pi % NSB) * (2 * PF_BN) + group * 32 + lane_off;
      if (!mbar_wait_bounded(&s_full[pi % P8_KBUF], (pi / P8_KBUF) & 1)) { ok = false; break; }
      tc::fence_after();
      uint32_t p[32];
#pragma unroll
      for (int c = 0; c < 16; ++c) p[16 + c] = 0u;
      float m_use = m_own, l_new = 0.f;
      bool agreed = false;
#pragma unroll 1
      for (;;) {
        // Block by block (one copy of the code: the roles share the instruction
        // caches): P under the reference m_use, its sum, and the largest score -- one
        // past the reference's reach is found only afterwards.
        const float mm = m_use == -INFINITY ? 0.f : m_use;   // -inf: nothing visible so far
        float mt = -INFINITY;
        l_new = 0.f;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          uint32_t s[32];
          tc::ld32(tb + 64 * h, s);
          tc::wait_ld();
          const int first = key0 + 32 * h;
          if (first + 31 > limit) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (first + c > limit) s[c] = 0xFF800000u;
          }
          const float k = h ? k1 : k0;
          const float ev = (float)(h ? ev1 : ev0);
          const uint64_t kk = f32x2(k, k), cc = f32x2(ev - mm, ev - mm);
          uint64_t sum = f32x2(0.f, 0.f);
          float x[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 16; ++c) p[c] = p[16 + c];
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float a0 = __uint_as_float(s[2 * c]), a1 = __uint_as_float(s[2 * c + 1]);
            x[c & 1] = max3(x[c & 1], a0, a1);
            float d0, d1;
            unpack_f32x2(fma_f32x2(f32x2(a0, a1), kk, cc), d0, d1);
            const float p0 = fast_exp2(d0), p1 = fast_exp2(d1);
            sum = add_f32x2(sum, f32x2(p0, p1));
            p[16 + c] = pack_f16x2(p0, p1);
          }
          mt = fmaxf(mt, fmaf(fmaxf(x[0], x[1]), k, ev));   // k is positive
          float u, v;
          unpack_f32x2(sum, u, v);
          l_new = fmaf(u + v, two8(-(h ? ev1 : ev0)), l_new);
        }
        const bool over = __any_sync(0xffffffffu, mt > m_use + P8_TOP);
        if (agreed) break;
        // the reference after tile j - 1, the other group's
        float m_ref = -INFINITY;
        if (j > 0) {
          const int jp = j - 1;
          if (!mbar_wait_bounded(&m_bar[(jp & 1) * 4 + quarter], (jp >> 1) & 1)) { ok = false; break; }
          m_ref = s_m[r];
        }
        if (!over && !__any_sync(0xffffffffu, m_ref != m_use)) break;
        // it has moved, or moves now (O's rows with it): once more
        const bool need = mt > m_ref + P8_TOP;
        m_use = need ? mt - P8_SET : m_ref;
        if (__any_sync(0xffffffffu, need) && j > 0) {
          const float f = (need && m_ref != -INFINITY) ? fast_exp2(m_ref - m_use) : 1.f;
          if (!mbar_wait_bounded(&pv_done[(j - 1) % PVR], ((j - 1) / PVR) & 1)) {
            ok = false;
            break;
          }
          tc::fence_after();
#pragma unroll 1
          for (int c0 = 0; c0 < D; c0 += 32) {
            uint32_t o[32];
            tc::ld32(tO + c0 + lane_off, o);
            tc::wait_ld();
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            tc::st32(tO + c0 + lane_off, o);
          }
        }
        agreed = true;
      }
      if (!ok) break;
      s_m[r] = m_use;
      __syncwarp();
      if (lane == 0) mbar_arrive(&m_bar[group * 4 + quarter]);
      if (m_use != m_own) {
        l = m_own == -INFINITY ? 0.f : l * fast_exp2(m_own - m_use);
        m_own = m_use;
      }
      l += l_new;
      tc::st32(tb, p);
      tc::wait_st();
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::arrive_cluster(&pv_ready[j % PVR], 0);
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    s_ml[group * PF_BM + r] = make_float2(m_own, l);
  }

  // ---- O / l -> bf16 (one split) or the unnormalized partial (m, l, O); each
  // softmax group half of the columns -------------------------------------------------
  const bool all_ok = !__syncthreads_or(!ok);
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");   // the merge waits for the rest
  if (warp >= P8_SM_WARP0) {
    const P8Out out = *s_out;
    const int64_t row_at = s_row[r];
    if (PLAN && row_at >= 0 && group == 0)   // neutral
      for (int u = 1; u <= out.unused; ++u) {
        a.part_ml[(row_at + u) * 2 + 0] = -INFINITY;
        a.part_ml[(row_at + u) * 2 + 1] = 0.f;
      }
    if (ntiles == 0) {   // an empty history range: a neutral partial
      if (out.split && row_at >= 0) {
        if (group == 0) {
          a.part_ml[row_at * 2 + 0] = -INFINITY;
          a.part_ml[row_at * 2 + 1] = 0.f;
        }
        float4* const po = reinterpret_cast<float4*>(a.part_o + row_at * D + group * (D / 2));
        for (int c = 0; c < D / 8; ++c) po[c] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    } else if (all_ok &&
               __all_sync(0xffffffffu, mbar_wait_bounded(&pv_done[(ntiles - 1) % PVR],
                                                         ((ntiles - 1) / PVR) & 1))) {
      tc::fence_after();
      const float m = s_m[r];   // after the last tile
      float lsum = 0.f;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float2 v = s_ml[g * PF_BM + r];
        // no reference: a sum of zero, or NaN where every score was
        lsum = v.x == -INFINITY ? lsum + v.y : fmaf(v.y, fast_exp2(v.x - m), lsum);
      }
      if (out.split && row_at >= 0 && group == 0) {
        a.part_ml[row_at * 2 + 0] = lsum == lsum ? m : 0.f;   // NaN: not to be taken for an empty range
        a.part_ml[row_at * 2 + 1] = lsum;
      }
      const float inv = lsum != 0.f ? 1.f / lsum : 0.f;
      // The warp's 32 half rows go through shared memory (16-byte piece p of row r at
      // p ^ (r & 7)), so that a store writes whole lines; a row per thread took 3 us.
      const uint32_t tr = smem_u32(sm) + (warp - P8_SM_WARP0) * (32 * (D / 2) * 4);
      const int lg = (D == 256 ? 4 : 3) + out.split;   // 2^lg 16-byte pieces a half row
      const uint32_t mine = tr + (lane << (lg + 4));
#pragma unroll 1
      for (int c0 = 0; c0 < D / 2; c0 += 32) {
        uint32_t o[32];
        tc::ld32(tO + group * (D / 2) + c0 + lane_off, o);
        tc::wait_ld();
        if (out.split) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            st_shared_v4(mine + (((c0 / 4 + k) ^ (lane & 7)) << 4), o[4 * k], o[4 * k + 1],
                         o[4 * k + 2], o[4 * k + 3]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              w[i] = pack_bf16x2_rn(__uint_as_float(o[8 * k + 2 * i]) * inv,
                                    __uint_as_float(o[8 * k + 2 * i + 1]) * inv);
            st_shared_v4(mine + (((c0 / 8 + k) ^ (lane & 7)) << 4), w[0], w[1], w[2], w[3]);
          }
        }
      }
      __syncwarp();
      const int row_bytes = out.split ? D * 4 : D * 2;
      uint8_t* const to = out.to + group * (row_bytes / 2);
#pragma unroll 4
      for (int i = lane; i < 32 << lg; i += 32) {
        const int row = i >> lg, piece = i & ((1 << lg) - 1);
        const int64_t dst = s_row[quarter * 32 + row];
        const uint4 v = ld_shared_v4(tr + (row << (lg + 4)) + ((piece ^ (row & 7)) << 4));
        if (dst >= 0)
          *reinterpret_cast<uint4*>(to + dst * row_bytes + piece * 16) = v;
      }
    } else if (all_ok && lane == 0) {
      flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
  }

  // neither CTA may release TMEM or exit while its partner can still reach it
  tc::fence_before();
  __syncthreads();
  tc::cluster_sync();
  if (warp == 0) {
    tc::fence_after();
    tc::dealloc2(*tmem_slot, 512);
  }
  if (warp >= P8_SM_WARP0 && all_ok && s_nan[D] != 0x7FFFFFFF) {   // NaN that some rows see
    const P8Out out = *s_out;
    const int64_t row_at = s_row[r];
    const int limit = s_lim[r];
    for (int d = group * (D / 2); d < (group + 1) * (D / 2) && row_at >= 0; ++d)
      if (s_nan[d] <= limit) {
        if (out.split)
          reinterpret_cast<float*>(out.to)[row_at * D + d] = __uint_as_float(0x7FC00000u);
        else
          reinterpret_cast<uint16_t*>(out.to)[row_at * D + d] = 0x7FC0u;
      }
  }
}

// The plan's estimate, in history tiles (0.8 us each at D = 256): a part beyond a
// place's first costs P8_HDR tiles (queries, pipeline fill, its partial rows), the
// merge P8_MERGE.  The tail is cut where that is sooner than one wave more.  2,048
// queries after 30,720 positions (44 of 196 pairs left over), side by side: uncut 1,055 us,
// cut 972 (967 to 974 with headers of 6 to 32; in other runs up to 1,005); with an earlier kernel uncut 1,243, the
// left-over pairs as a second launch of three even splits 1,163, cut so 1,131.
constexpr int P8_HDR = 12, P8_MERGE = 16, P8_MIN_PIECE = 16;

void kv8_prefill_plan(int64_t G, int64_t Hkv, int64_t q_start, int64_t chunk_len, bool causal,
                      int64_t num_sms, P8Plan* plan) {
  plan->whole = plan->n = plan->rows = 0;
  plan->k = 1;
  if (G < 1 || G > PF_BM || Hkv < 1 || num_sms < 2 || chunk_len < 1 || q_start < 4 * chunk_len)
    return;   // pairs of unlike lengths already end one after the other
  const int64_t slots = num_sms / 2 < P8_MAX_SEG / 2 ? num_sms / 2 : P8_MAX_SEG / 2;
  const int64_t qpp = 2 * (PF_BM / G);                  // queries per CTA pair
  const int64_t pph = (chunk_len + qpp - 1) / qpp;      // pairs per KV head
  const int64_t pairs = pph * Hkv, rem = pairs % slots;
  if (pairs <= slots || rem == 0 || pairs > 0xFFFF) return;
  const int64_t t_tail = (rem + Hkv - 1) / Hkv, tail = t_tail * Hkv;
  if (t_tail >= pph || tail > slots) return;
  // pair p of the launch order holds query tiles pph - 1 - p / Hkv of its head
  auto tiles_of = [&](int64_t p) {
    const int64_t q = (pph - p / Hkv) * qpp;
    const int64_t seen = causal ? q_start + (q < chunk_len ? q : chunk_len) : q_start + chunk_len;
    return (seen + PF_BN - 1) / PF_BN;
  };
  const int64_t first = pairs - tail;
  int64_t total = 0;
  for (int64_t p = first; p < pairs; ++p) total += tiles_of(p) + P8_HDR;
  int64_t width = (total + slots - 1) / slots;
  if (width < P8_MIN_PIECE + P8_HDR) width = P8_MIN_PIECE + P8_HDR;
  if (width + P8_MERGE >= tiles_of(first)) return;
  int n = 0, k = 1;
  int64_t len[P8_MAX_SEG];
  int64_t at = 0;   // where the pair's run (header, then tiles) begins
  for (int64_t p = first; p < pairs; ++p) {
    const int64_t nt = tiles_of(p), end = at + P8_HDR + nt;
    int64_t t0 = 0;
    int z = 0;
    while (t0 < nt) {
      // up to the next cut; what is shorter than a header is not worth a part
      const int64_t here = at + P8_HDR + t0;
      int64_t cut = (here / width + 1) * width;
      if (cut - here < P8_HDR) cut += width;
      const int64_t t1 = end - cut < P8_HDR ? nt : cut - at - P8_HDR;
      if (n == P8_MAX_SEG || z == 255) return;
      int i = n++;
      for (; i > 0 && len[i - 1] < t1 - t0; --i) {   // longest first
        len[i] = len[i - 1];
        plan->seg[i] = plan->seg[i - 1];
      }
      len[i] = t1 - t0;
      plan->seg[i] = P8Seg{(uint16_t)p, (uint8_t)z, (uint8_t)(t1 == nt),
                           (uint16_t)((t0 * 32768 + nt - 1) / nt),
                           (uint16_t)(t1 == nt ? 32768 : (t1 * 32768 + nt - 1) / nt)};
      ++z;
      t0 = t1;
    }
    if (z > k) k = z;
    at = end;
  }
  plan->whole = (int32_t)first;
  plan->rows = (int32_t)(t_tail * qpp);
  plan->k = k;
  plan->n = n;
}

template <int D, bool PLAN>
static int launch_t(const CUtensorMap& kmap, const PrefillArgs& a,
                    const typename P8PlanArg<PLAN>::type& plan, const dim3& grid,
                    cudaStream_t stream) {
  const auto kernel = kv8_prefill_kernel<D, PLAN>;
  if (smem_optin((const void*)kernel, P8Smem<D>::TOTAL) != JF_OK) return JF_ERR_CUDA;
  // programmatic dependent launch: barriers and TMEM are set up while the kernel before drains
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(P8_THREADS);
  cfg.dynamicSmemBytes = P8Smem<D>::TOTAL;
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, kmap, a, plan) == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

int launch_kv8_prefill(const Geom& g, const jf_kv_pool& pool, const PrefillArgs& a,
                       const P8Plan* plan, unsigned ctas, unsigned splits, cudaStream_t stream) {
  CUtensorMap kmap;
  const int st = kv8_tensor_map(g, pool.base, 1, 32, 1, &kmap);
  if (st) return st;
  const dim3 grid(ctas, 1u, splits);
  if (plan)
    return g.D == 256 ? launch_t<256, true>(kmap, a, *plan, grid, stream)
                      : launch_t<128, true>(kmap, a, *plan, grid, stream);
  return g.D == 256 ? launch_t<256, false>(kmap, a, P8NoPlan{}, grid, stream)
                    : launch_t<128, false>(kmap, a, P8NoPlan{}, grid, stream);
}

}  // namespace jfkv
