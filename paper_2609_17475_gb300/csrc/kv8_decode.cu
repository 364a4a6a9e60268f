// Single-token attention over the 8-bit block-scaled cache, with the
// attention weights each position draws added up on request.
//
// Split kernel.  One 12-warp CTA per SM takes an equal piece of the batch's
// positions (of one KV head); its warps take the piece's 16-position chunks
// in turn, each through a private ring of shared-memory stages that one TMA
// copy per chunk fills: K and V rows of 16 positions, as [K|V][16 positions]
// [D/128][128 bytes], 128-byte swizzle.
//  * S^T = K q^T: A = K codes [16 positions x 16 d], B = q [16 d x 8 heads].
//    The four lanes of a position read 16 bytes each and every word's four
//    codes become two f16x2 operands (exact: e4m3 lies inside fp16), the order
//    of d inside a k-step being free as long as q follows it.  The K block's
//    scale multiplies the fp32 score.
//  * O^T += V^T P^T: A = V codes [16 d x 16 positions]: a lane reads 16 d of
//    four positions, two byte permutes and four conversions give the four A
//    registers; B = P (the score registers transposed with movmatrix).
//  * Scales are powers of two, so the V block's scale costs nothing: with
//    y_t = x_t + e_t (x_t the log2-domain score, e_t the V exponent),
//      sum_t 2^x_t V_t = sum_t 2^(y_t - m) code_t * 2^m,
//      sum_t 2^x_t     = sum_t 2^(y_t - m) 2^-e_t * 2^m
//    for any reference m; y_t - m <= 14 keeps 2^(y - m) inside fp16 and far
//    above its subnormals, whatever the blocks' scales are.  m moves only when
//    y exceeds it by more than 14 (to 10 below the new largest).
//  * MMA rows are dealt to the chunk's positions, and V's 16-byte pieces to
//    lanes, in an order (k8_pos, k8_vchunk) that keeps every 128-bit
//    shared-memory read of the swizzled tiles free of bank conflicts: the eight
//    lanes of a quarter-warp meet eight different 16-byte columns.
// Bound: reading the codes.  One request of 262,144 positions, 24 / 4 heads x 256: 88 us
// for 537 MB, 6.1 TB/s (0.90 of the copy rate), the merge 3 us of it; the split kernel
// moves 1.00 times those bytes.  32 requests of up to 65,535 positions with weights:
// 196 us, 158 at the copy rate, merging and weighing about 20.  One request of
// 4,096 (8 / 2 heads x 128): 8.5 us, two launches' latency.
// Rounding: q enters as fp16 after a power-of-two scale per head that puts
// its largest element in [2^13, 2^14) (exact for elements within 2^27 of it);
// probabilities enter P V as fp16 (11 bits); sums are fp32.
//
// Merge kernel.  Joins the pieces' partials of each query row:
//   o = sum_s 2^(m_s - m) O_s / l,  l = sum_s 2^(m_s - m) l_s.
// Weights.  Where they are asked for, the split kernel leaves the scores x in the
// workspace (they mostly stay in L2), and CTAs beside the merge's add
//   weights_out[b, h, t] = weights_in[b, h, t] + sum_g 2^(x_gt - m_g) / l_g.
// Scores lie as [chunk of 16 positions][8 positions of it][odd heads or even]
// [pair of heads][8 positions], as the MMA leaves them, so that each store of
// the split kernel is one run of 32 bytes a pair of heads.
#include <cmath>

#include "kv8.cuh"

namespace jfkv {

int sm_count();

constexpr int K8_CH = 32;       // positions per plan chunk
constexpr int K8_SUB = 16;      // positions per pipeline stage
constexpr int K8_NW = 12;       // warps per CTA, one CTA per SM (two of 6 warps share the SM
                                // unevenly: one request of 262,144 positions 103 us, not 88)
// plan places standing for a segment's start (32 requests to 65,535 with weights, with 8,
// 16, 24, 32 and 48: 206, 200, 196, 196 and 196 us; 16 to 9,000 positions, 4 heads x 128:
// 17.1, 17.2, 17.4, 18.9 and 17.9)
constexpr int K8_HDR = 24;
constexpr int K8_MIN_W = 6;     // least places per piece (one stage for each warp)
constexpr float K8_TOP = 14.f;  // 2^(y - m) stays below 2^14
constexpr float K8_SET = 10.f;  // a new m puts the largest y at 2^10

struct Kv8DecodeArgs {
  const uint8_t* pool;
  int64_t num_pages;
  int64_t page_bytes;
  int64_t codes_region;
  int64_t sb_region;
  int32_t P, log2P, Hkv, Hq, G, B;
  const int32_t* page_table;
  int32_t pt_stride;
  const int32_t* ctx;
  const uint16_t* q;
  uint16_t* out;
  float* part_ml;
  float* part_o;
  int32_t* status;
  int32_t budget;           // pieces per KV head
  float scale_log2;
  float* scores;            // [B, Hkv] blocks of sstride floats (above), or null
  int64_t sstride;          // chunks of 16 positions x 32 x pairs
  int32_t pairs;            // pairs of a KV head's query heads: ceil(G / 2)
  const float* w_in;        // [B, Hkv, wstride] or null (zeros)
  float* w_out;
  int64_t wstride;
  int32_t slices;           // merging CTAs per query row
  int32_t wtiles, wsteps;   // weighing CTAs per (request, KV head), steps of each
};

// ---- plan: the requests' 32-position chunks laid end to end, each request's
// run preceded by K8_HDR places for its segment's start, cut into `budget`
// pieces of W places.  Piece x's segment of request b is partial row x + b
// (along the sequence every boundary advances x + b, so rows never repeat
// and a request's are consecutive).
__device__ __forceinline__ int k8_ctx(const Kv8DecodeArgs& a, int b) {
  const int64_t cap = (int64_t)a.pt_stride * a.P;
  const int64_t c = a.ctx[b];
  return (int)(c < 0 ? 0 : (c > cap ? cap : c));
}
__device__ __forceinline__ int k8_run(const Kv8DecodeArgs& a, int b) {
  const int n = (int)(((int64_t)k8_ctx(a, b) + K8_CH - 1) / K8_CH);
  return n > 0 ? n + K8_HDR : 0;
}
__device__ long long k8_total(const Kv8DecodeArgs& a, int lane) {
  long long T = 0;
  for (int b = lane; b < a.B; b += 32) T += k8_run(a, b);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) T += __shfl_xor_sync(0xffffffffu, T, o);
  return T;
}
__device__ __forceinline__ long long k8_width(const Kv8DecodeArgs& a, long long T) {
  const long long w = (T + a.budget - 1) / a.budget;
  return w < K8_MIN_W ? K8_MIN_W : w;
}
struct K8Hit {
  int b;             // request, -1: none
  long long start;   // its first place
  int n;             // its places
};
// the request that holds place `pos`, or with pos < 0 request want; whole warp
__device__ K8Hit k8_find(const Kv8DecodeArgs& a, long long pos, int want, int lane) {
  long long base = 0;
  for (int b0 = 0; b0 < a.B; b0 += 32) {
    const int b = b0 + lane;
    const int n = b < a.B ? k8_run(a, b) : 0;
    long long incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const long long excl = base + incl - n;
    const bool hit = pos >= 0 ? (n > 0 && pos >= excl && pos < excl + n) : b == want;
    const unsigned m = __ballot_sync(0xffffffffu, hit);
    if (m) {
      const int src = __ffs(m) - 1;
      return K8Hit{b0 + src, __shfl_sync(0xffffffffu, excl, src),
                   __shfl_sync(0xffffffffu, n, src)};
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  return K8Hit{-1, 0, 0};
}

template <int D>
struct K8Smem {
  static constexpr int STAGES = D == 256 ? 2 : 4;
  static constexpr int KV = K8_SUB * D;              // bytes of K (or V) of a stage
  static constexpr int STAGE = 2 * KV;
  static constexpr int WARP = STAGES * STAGE;        // one warp's ring
  static constexpr int RING = K8_NW * WARP;
  static constexpr int SROW = D + 4;                 // padded fp32 row of the combine
  static constexpr int OFF_ML = RING;                // [warp][8] (m, l)
  static constexpr int OFF_BAR = OFF_ML + K8_NW * 8 * 8;
  static constexpr int TOTAL = OFF_BAR + K8_NW * STAGES * 8;
  static_assert(8 * SROW * 4 <= WARP, "a warp's output rows fit its ring");
  static_assert(TOTAL <= 227 * 1024, "shared memory per CTA");
};

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}

// Byte offset of 16-byte piece `ch` of 128-byte half `h` of position `pos` in
// a stage's K (or V) tile: rows of 128 bytes, the piece index xor-ed with the
// row's low three bits.
template <int D>
__device__ __forceinline__ uint32_t k8_at(int pos, int h, int ch) {
  return pos * D + h * 128 + ((uint32_t)(ch ^ ((pos * (D / 128) + h) & 7)) << 4);
}
// Position (of 8) of MMA row m.  K reads take rows 2q, 2q + 1 in one quarter-
// warp: their swizzles differ in bit 2.  V reads take rows 0, 2, 4, 6 (or 1, 3,
// 5, 7) for four lanes and two adjacent pieces: their swizzles differ in the
// two bits that k8_vchunk's pieces share.
template <int D>
__device__ __forceinline__ int k8_pos(int m) {
  return D == 256 ? ((m & 1) ? ((m >> 1) ^ 2) + 4 : m >> 1) : (m >> 1) | ((m & 1) << 2);
}
template <int D>
__device__ __forceinline__ int k8_vchunk(int r) {
  return D == 256 ? r : (r >> 1) | ((r & 1) << 2);
}

template <int D>
struct K8State {
  float m0, m1, l0, l1;          // heads 2c, 2c + 1
  float O[D / 128][8][4];        // [half][pair j]: d = 16 chunk + 2j (+1), heads 2c, 2c + 1
};

// One stage of 16 positions.  FULL: all of them are attended; otherwise those
// at or past nv are not, and nothing of their bytes is used.
template <int D, bool FULL>
__device__ __forceinline__ void k8_chunk(K8State<D>& st, const uint32_t (&qf)[D / 16][2],
                                         uint32_t kb, int r, int c, float cA0, float cA1,
                                         float ks, float ve, float vinv, int nv, float* sc,
                                         int pairs, bool h0, bool h1) {
  constexpr int HV = D / 128;
  constexpr float NEG = -INFINITY;
  const int pr = k8_pos<D>(r);       // position of MMA row r; row r + 8: pr + 8
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  float s2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < HV; ++h)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const uint32_t off = kb + k8_at<D>(pr, h, 4 * kk + c);
      const uint4 ka = lds128(off), kc = lds128(off + 8 * D);   // 8 positions on: same swizzle
      const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wc[4] = {kc.x, kc.y, kc.z, kc.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t a0, a1, a2, a3;
        f16x4_of_e4m3(wa[w], a0, a2);
        f16x4_of_e4m3(wc[w], a1, a3);
        const int ki = (h * 2 + kk) * 4 + w;
        mma_f16((w & 1) ? s2 : s, a0, a1, a2, a3, qf[ki][0], qf[ki][1]);
      }
    }
  const float f0 = cA0 * ks, f1 = cA1 * ks;
  float x[4];
  x[0] = (s[0] + s2[0]) * f0;
  x[1] = (s[1] + s2[1]) * f1;
  x[2] = (s[2] + s2[2]) * f0;
  x[3] = (s[3] + s2[3]) * f1;
  const bool va = FULL || pr < nv, vb = FULL || pr + 8 < nv;
  if (sc) {   // this stage's scores (log2 domain) of this thread's heads, if they exist
    sc += pr;
    if (h0 && va) sc[0] = x[0];
    if (h1 && va) sc[8 * pairs] = x[1];
    if (h0 && vb) sc[16 * pairs] = x[2];
    if (h1 && vb) sc[24 * pairs] = x[3];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (i < 2 ? va : vb) ? x[i] + ve : NEG;
  const float t0 = fmaxf(x[0], x[2]), t1 = fmaxf(x[1], x[3]);
  if (__any_sync(0xffffffffu, t0 > st.m0 + K8_TOP || t1 > st.m1 + K8_TOP)) {
    float g0 = t0, g1 = t1;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      g0 = fmaxf(g0, __shfl_xor_sync(0xffffffffu, g0, o));
      g1 = fmaxf(g1, __shfl_xor_sync(0xffffffffu, g1, o));
    }
    const float n0 = g0 > st.m0 + K8_TOP ? g0 - K8_SET : st.m0;
    const float n1 = g1 > st.m1 + K8_TOP ? g1 - K8_SET : st.m1;
    const float e0 = st.m0 == NEG ? 0.f : fast_exp2(st.m0 - n0);
    const float e1 = st.m1 == NEG ? 0.f : fast_exp2(st.m1 - n1);
    st.m0 = n0;
    st.m1 = n1;
    st.l0 *= e0;
    st.l1 *= e1;
#pragma unroll
    for (int h = 0; h < HV; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        st.O[h][j][0] *= e0;
        st.O[h][j][1] *= e1;
        st.O[h][j][2] *= e0;
        st.O[h][j][3] *= e1;
      }
  }
  float p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = fast_exp2(x[i] - ((i & 1) ? st.m1 : st.m0));
    if (!FULL && x[i] == NEG) p[i] = 0.f;   // also where the row has seen nothing (m = -inf)
  }
  st.l0 = fmaf(p[0] + p[2], vinv, st.l0);
  st.l1 = fmaf(p[1] + p[3], vinv, st.l1);
  const uint32_t b0 = movm_t(pack_f16x2(p[0], p[1]));
  const uint32_t b1 = movm_t(pack_f16x2(p[2], p[3]));
  const uint32_t vb0 = kb + K8_SUB * D;
#pragma unroll
  for (int h = 0; h < HV; ++h) {
    // 16 d of the positions of MMA columns 2c, 2c + 1, 2c + 8, 2c + 9
    uint32_t v[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pos = k8_pos<D>(2 * c + (i & 1)) + 8 * (i >> 1);
      uint4 t = lds128(vb0 + k8_at<D>(pos, h, k8_vchunk<D>(r)));
      if (!FULL && pos >= nv) t = make_uint4(0u, 0u, 0u, 0u);
      v[i][0] = t.x;
      v[i][1] = t.y;
      v[i][2] = t.z;
      v[i][3] = t.w;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t sel = e ? 0x7362u : 0x5140u;
        uint32_t a0, a1, a2, a3;
        f16x4_of_e4m3(__byte_perm(v[0][w], v[1][w], sel), a0, a1);
        f16x4_of_e4m3(__byte_perm(v[2][w], v[3][w], sel), a2, a3);
        mma_f16(st.O[h][2 * w + e], a0, a1, a2, a3, b0, b1);
      }
  }
}

template <int D, bool WEIGH>
__global__ void __launch_bounds__(K8_NW * 32, 1)
kv8_split_kernel(const __grid_constant__ CUtensorMap tmap, const Kv8DecodeArgs a) {
  using L = K8Smem<D>;
  constexpr int ST = L::STAGES;
  constexpr int HV = D / 128;
  constexpr float NEG = -INFINITY;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* const bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = lane >> 2, c = lane & 3;
  const int kvh = blockIdx.y;
  const bool aligned = (smem_u32(smem) & 1023) == 0;
  if (aligned) {
    if (threadIdx.x == 0) prefetch_tensormap(&tmap);
    if (lane == 0) {
      for (int s = 0; s < ST; ++s) mbar_init(&bars[warp * ST + s], 1);
      fence_barrier_init();
    }
  }
  __syncwarp();
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (!aligned) {
    if (threadIdx.x == 0) flag_error(a.status, JF_DEV_ERR_LAYOUT);
    return;
  }
  const uint32_t ring = smem_u32(smem) + warp * L::WARP;
  const uint64_t l2pol = l2_evict_first_policy();
  const long long T = k8_total(a, lane);
  const long long W = k8_width(a, T);
  long long pos = (long long)blockIdx.x * W;
  const long long end = min(pos + W, T);
  uint32_t used = 0;   // stages this warp has gone through (ring position and phase)
  while (pos < end) {
    const K8Hit hit = k8_find(a, pos, -1, lane);
    if (hit.b < 0) break;
    const int b = hit.b;
    const int u0 = (int)(pos - hit.start);
    const int u1 = (int)(min(end, hit.start + hit.n) - hit.start);
    const int ctx = k8_ctx(a, b);
    // this segment's stages [s0, s1) of 16 positions
    const int s0 = max(u0 - K8_HDR, 0) * 2;
    const int s1 = min(max(u1 - K8_HDR, 0) * 2, (int)((ctx + (int64_t)K8_SUB - 1) / K8_SUB));
    const int n_cta = max(s1 - s0, 0);
    const int my_n = n_cta > warp ? (n_cta - warp + K8_NW - 1) / K8_NW : 0;
    auto pos_of = [&](int it) { return (s0 + warp + it * K8_NW) * K8_SUB; };

    // page ids: lane i holds that of this warp's stage 32k + i
    auto load_pages = [&](int blk) -> int {
      const int it = blk * 32 + lane;
      return it < my_n ? __ldg(a.page_table + (int64_t)b * a.pt_stride + (pos_of(it) >> a.log2P))
                       : -1;
    };
    int pg_cur = load_pages(0), pg_next = load_pages(1);
    float ksc[ST], vsc[ST];   // scales of the stages in flight
    uint32_t valid = 0;
    auto issue = [&](int it, int s) {
      if (it >= 32 && (it & 31) == 0) {
        pg_cur = pg_next;
        pg_next = load_pages((it >> 5) + 1);
      }
      const int page = __shfl_sync(0xffffffffu, pg_cur, it & 31);
      const bool ok = page >= 0 && page < a.num_pages;
      const int slot = pos_of(it) & (a.P - 1);
      const int rs = (used + it) % ST;
      uint64_t* const bar = &bars[warp * ST + rs];
      if (lane == 0) {
        if (!ok) {
          flag_error(a.status, JF_DEV_ERR_PAGE_ID);
          mbar_arrive(bar);
        } else {
          mbar_arrive_expect_tx(bar, L::STAGE);
          tma_load_5d_hint(smem + warp * L::WARP + rs * L::STAGE, &tmap, 0, 0, kvh * a.P + slot, 0,
                           page, bar, l2pol);
        }
      }
      ksc[s] = vsc[s] = 1.f;
      if (ok) {
        const float* sc = reinterpret_cast<const float*>(a.pool + (int64_t)page * a.page_bytes +
                                                         2 * a.codes_region) +
                          kvh * (a.P / KV8_BLOCK) + slot / KV8_BLOCK;
        ksc[s] = sc[0];   // written by an append that this grid may overlap: no read-only load
        vsc[s] = sc[a.sb_region / 4];
      }
      valid = (valid & ~(1u << s)) | ((uint32_t)ok << s);
    };
#pragma unroll
    for (int s = 0; s < ST; ++s)
      if (s < my_n) issue(s, s);

    // ---- query: fragments of head r, scaled by a power of two ----------------
    uint32_t qf[D / 16][2];
    float cA0, cA1;
    {
      const bool head_ok = r < a.G;
      const uint16_t* qrow = a.q + ((int64_t)b * a.Hq + kvh * a.G + (head_ok ? r : 0)) * D;
      uint4 qv[D / 64][2];
      uint32_t mx = 0;   // largest magnitude's bf16 bits
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          qv[i][e] = head_ok ? *reinterpret_cast<const uint4*>(qrow + 64 * i + 16 * c + 8 * e)
                             : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t w[4] = {qv[i][e].x, qv[i][e].y, qv[i][e].z, qv[i][e].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mx = max(mx, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
        }
      mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      // largest element in [2^13, 2^14); a subnormal or zero row: times 2^100
      const int qe = mx >= 0x80u ? max((int)(mx >> 7) - 127 - 13, -100) : -100;
      const float qs = two8(-qe);
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t w[4] = {qv[i][e].x, qv[i][e].y, qv[i][e].z, qv[i][e].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            qf[4 * i + 2 * e + (k >> 1)][k & 1] =
                pack_f16x2(bf16lo_to_f32(w[k]) * qs, bf16hi_to_f32(w[k]) * qs);
        }
      // a head with an infinity or a NaN is NaN by its factor, whatever the keys
      const float mine = mx >= 0x7F80u ? __uint_as_float(0x7FC00000u) : a.scale_log2 * two8(qe);
      cA0 = __shfl_sync(0xffffffffu, mine, 8 * c);       // lane of head 2c: r = 2c, c = 0
      cA1 = __shfl_sync(0xffffffffu, mine, 8 * c + 4);
    }
    float* scb = nullptr;   // this thread's pair of heads in the segment's scores
    if constexpr (WEIGH) scb = a.scores + ((int64_t)b * a.Hkv + kvh) * a.sstride + 8 * c;

    K8State<D> st;
    st.m0 = st.m1 = NEG;
    st.l0 = st.l1 = 0.f;
#pragma unroll
    for (int h = 0; h < HV; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.O[h][j][i] = 0.f;

    int done = 0;
    for (int it0 = 0; it0 < my_n; it0 += ST) {
#pragma unroll
      for (int s = 0; s < ST; ++s) {
        const int it = it0 + s;
        if (it < my_n && done == it) {
          const int rs = (used + it) % ST;
          if (__all_sync(0xffffffffu,
                         mbar_wait_bounded(&bars[warp * ST + rs], ((used + it) / ST) & 1))) {
            done = it + 1;
            const int p0 = pos_of(it);
            // positions of this stage that are attended; a score row holds
            // wstride of them
            int lim = ctx;
            if constexpr (WEIGH) lim = (int)min((int64_t)ctx, a.wstride);
            const int nv = ((valid >> s) & 1u) ? lim - p0 : 0;
            const int ek = exp8_of_scale(ksc[s]), ev = exp8_of_scale(vsc[s]);
            const uint32_t kb = ring + rs * L::STAGE;
            float* sc = nullptr;
            if constexpr (WEIGH) {
              sc = scb + (int64_t)(p0 / K8_SUB) * (32 * a.pairs);
              if (!((valid >> s) & 1u) && p0 < lim) {   // a page outside the pool: no weight
                const int pr = k8_pos<D>(r);
                if (2 * c < a.G) sc[pr] = sc[pr + 16 * a.pairs] = NEG;
                if (2 * c + 1 < a.G) sc[pr + 8 * a.pairs] = sc[pr + 24 * a.pairs] = NEG;
              }
            }
            if (nv >= K8_SUB)
              k8_chunk<D, true>(st, qf, kb, r, c, cA0, cA1, two8(ek), (float)ev, two8(-ev), 0, sc,
                                a.pairs, 2 * c < a.G, 2 * c + 1 < a.G);
            else
              k8_chunk<D, false>(st, qf, kb, r, c, cA0, cA1, two8(ek), (float)ev, two8(-ev), nv, sc,
                                 a.pairs, 2 * c < a.G, 2 * c + 1 < a.G);
            __syncwarp();
            if (it + ST < my_n) {
              fence_proxy_async_smem();
              issue(it + ST, s);
            }
          }
        }
      }
      if (done < min(it0 + ST, my_n)) break;
    }
    const bool gave_up = done < my_n;
    if (gave_up) {
      if (lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
      for (int it = done; it < my_n && it < done + ST; ++it)   // copies still in flight
        mbar_wait_bounded(&bars[warp * ST + (used + it) % ST], ((used + it) / ST) & 1, 1u << 16);
    }
    used += my_n;

    // ---- combine the warps and write the segment's partial --------------------
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      st.l0 += __shfl_xor_sync(0xffffffffu, st.l0, o);
      st.l1 += __shfl_xor_sync(0xffffffffu, st.l1, o);
    }
    {
      float* const so = reinterpret_cast<float*>(smem + warp * L::WARP);
      float2* const sml = reinterpret_cast<float2*>(smem + L::OFF_ML) + warp * 8;
      const int vc = k8_vchunk<D>(r);
#pragma unroll
      for (int h = 0; h < HV; ++h)
#pragma unroll
        for (int j = 0; j < 8; j += 2)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            *reinterpret_cast<float4*>(so + (2 * c + hh) * L::SROW + h * 128 + vc * 16 + 2 * j) =
                make_float4(st.O[h][j][hh], st.O[h][j][2 + hh], st.O[h][j + 1][hh],
                            st.O[h][j + 1][2 + hh]);
      if (r == 0) {
        sml[2 * c] = make_float2(st.m0, st.l0);
        sml[2 * c + 1] = make_float2(st.m1, st.l1);
      }
    }
    if (__syncthreads_or(gave_up)) return;
    const int64_t row0 = ((int64_t)blockIdx.x + b) * a.Hq + kvh * a.G;
    for (int i = threadIdx.x; i < a.G * (D / 4); i += K8_NW * 32) {
      const int g = i / (D / 4), d = 4 * (i % (D / 4));
      const float2* const sml = reinterpret_cast<const float2*>(smem + L::OFF_ML) + g;
      float M = NEG;
#pragma unroll
      for (int w = 0; w < K8_NW; ++w) M = fmaxf(M, sml[w * 8].x);
      float lsum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < K8_NW; ++w) {
        const float2 ml = sml[w * 8];
        // no reference: this warp saw no position (l and O are zero), or NaN scores alone
        const float f = ml.x == NEG ? ml.y : fast_exp2(ml.x - M);
        const float4 o = *reinterpret_cast<const float4*>(
            reinterpret_cast<const float*>(smem + w * L::WARP) + g * L::SROW + d);
        lsum = fmaf(f, ml.y, lsum);
        acc.x = fmaf(f, o.x, acc.x);
        acc.y = fmaf(f, o.y, acc.y);
        acc.z = fmaf(f, o.z, acc.z);
        acc.w = fmaf(f, o.w, acc.w);
      }
      *reinterpret_cast<float4*>(a.part_o + (row0 + g) * D + d) = acc;
      if (d == 0) *reinterpret_cast<float2*>(a.part_ml + (row0 + g) * 2) = make_float2(M, lsum);
    }
    pos = hit.start + u1;
    if (pos < end) {   // the ring is free for the next segment's copies
      __syncthreads();
      fence_proxy_async_smem();
    }
  }
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
}

// partial rows of request b: row .. row + n - 1 (times Hq); whole warp
struct K8Rows {
  int row, n;
};
__device__ K8Rows k8_rows(const Kv8DecodeArgs& a, int b, int lane) {
  const long long W = k8_width(a, k8_total(a, lane));
  const K8Hit h = k8_find(a, -1, b, lane);
  if (h.n <= 0) return K8Rows{0, 0};
  const int x0 = (int)(h.start / W), x1 = (int)((h.start + h.n - 1) / W);
  return K8Rows{x0 + b, x1 - x0 + 1};
}

constexpr int K8F_THREADS = 256;
constexpr int K8F_COLS = 64;                       // columns of an output row per merging step

constexpr int K8W_STEP = 4 * K8F_THREADS;   // positions a weighing CTA takes at once: 4 a thread

// Weights of positions t0 .. of a (request, KV head): weights_in plus 2^(x - m) / l over
// its heads, m and l from the pieces' partials (warp g those of head g), so that nothing
// waits for the merge.
__device__ void k8_weigh(const Kv8DecodeArgs& a, int tile, int kvh, int b, float2* head_ml,
                         int* plan) {
  constexpr float NEG = -INFINITY;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = (int)min((int64_t)k8_ctx(a, b), a.wstride);
  const int64_t t0 = (int64_t)tile * (a.wsteps * K8W_STEP);
  if (t0 >= n) return;   // the whole CTA
  // a thread takes four adjacent positions a step; the heads' scores are all
  // loaded before any is used, the first step's before m and l are known
  const float* const sc = a.scores + ((int64_t)b * a.Hkv + kvh) * a.sstride;
  const int64_t wrow = ((int64_t)b * a.Hkv + kvh) * a.wstride;
  auto at = [&](int step) { return (int)t0 + step * K8W_STEP + (int)threadIdx.x * 4; };
  float4 x[8];
  auto load = [&](int t) {
    const float* const sx = sc + (int64_t)(t / K8_SUB) * (32 * a.pairs) +
                            ((t >> 3) & 1) * (16 * a.pairs) + (t & 7);
#pragma unroll
    for (int g = 0; g < 8; ++g)
      if (g < a.G)
        x[g] = __ldcs(reinterpret_cast<const float4*>(sx + ((g & 1) * a.pairs + (g >> 1)) * 8));
  };
  if (at(0) < n) load(at(0));
  if (warp == 0) {
    const K8Rows r = k8_rows(a, b, lane);
    if (lane == 0) {
      plan[0] = r.row;
      plan[1] = r.n;
    }
  }
  __syncthreads();
  if (warp < a.G) {
    const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) +
                             (int64_t)plan[0] * a.Hq + kvh * a.G + warp;
    float M = NEG, l = 0.f;
    for (int s = lane; s < plan[1]; s += 32) M = fmaxf(M, ml[(int64_t)s * a.Hq].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    for (int s = lane; s < plan[1]; s += 32) {
      const float2 v = ml[(int64_t)s * a.Hq];
      l = fmaf(v.x == NEG ? v.y : fast_exp2(v.x - M), v.y, l);   // v.y is 0 or NaN there
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    // nothing attended: scores of -inf and weights of zero
    if (lane == 0) head_ml[warp] = make_float2(M == NEG ? 0.f : M, l != 0.f ? 1.f / l : 0.f);
  }
  __syncthreads();
#pragma unroll 1
  for (int step = 0; step < a.wsteps; ++step) {
    const int t = at(step);
    if (t >= n) return;
    float w[4], add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a.w_in && t + i < n ? a.w_in[wrow + t + i] : 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g)
      if (g < a.G) {
        const float2 m = head_ml[g];
        add[0] = fmaf(fast_exp2(x[g].x - m.x), m.y, add[0]);
        add[1] = fmaf(fast_exp2(x[g].y - m.x), m.y, add[1]);
        add[2] = fmaf(fast_exp2(x[g].z - m.x), m.y, add[2]);
        add[3] = fmaf(fast_exp2(x[g].w - m.x), m.y, add[3]);
      }
    if (step + 1 < a.wsteps && at(step + 1) < n) load(at(step + 1));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t + i < n) a.w_out[wrow + t + i] = w[i] + add[i];
  }
}

// A CTA takes one query row, every `slices`-th run of 64 columns of it; warp w
// sums the partials w, w + 8, ... of two columns a lane.  WEIGH: the first CTAs
// weigh (a kernel of its own after the merge: one request of 5,000 positions 11.6 us,
// not 8.7; 32 mixed requests, then, 207, not 205).
template <int D, bool WEIGH>
__global__ void __launch_bounds__(K8F_THREADS) kv8_merge_kernel(const Kv8DecodeArgs a) {
  constexpr float NEG = -INFINITY;
  __shared__ float2 red[8][32];
  __shared__ float red_l[8];
  __shared__ int plan[2];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  int cta = (int)blockIdx.x;
  if constexpr (WEIGH) {
    const int weighing = a.wtiles * a.Hkv * a.B;
    if (cta < weighing) {
      const int row = cta / a.wtiles;
      k8_weigh(a, cta - row * a.wtiles, row % a.Hkv, row / a.Hkv, red[0], plan);
      return;
    }
    cta -= weighing;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml);
  const int sl0 = cta % a.slices;
  const int hq = (cta / a.slices) % a.Hq;
  const int b = cta / (a.slices * a.Hq);
  if (sl0 == 0 && hq == 0 && threadIdx.x == 0) {
    const int64_t ctx = a.ctx[b];
    if (ctx < 0 || ctx > (int64_t)a.pt_stride * a.P || (a.w_out && ctx > a.wstride))
      flag_error(a.status, JF_DEV_ERR_POSITION);
  }
  if (warp == 0) {   // one warp works the plan out
    const K8Rows r = k8_rows(a, b, lane);
    if (lane == 0) {
      plan[0] = r.row;
      plan[1] = r.n;
    }
  }
  __syncthreads();
  const K8Rows rows{plan[0], plan[1]};
  float M = NEG;
  for (int s = lane; s < rows.n; s += 32) M = fmaxf(M, ml[(int64_t)(rows.row + s) * a.Hq + hq].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  for (int sl = sl0; sl < D / K8F_COLS; sl += a.slices) {
    float l = 0.f;
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll 5
    for (int s = warp; s < rows.n; s += 8) {
      const int64_t row = (int64_t)(rows.row + s) * a.Hq + hq;
      const float2 v = ml[row];
      const float2 o =
          *reinterpret_cast<const float2*>(a.part_o + row * D + sl * K8F_COLS + 2 * lane);
      const float f = v.x == NEG ? v.y : fast_exp2(v.x - M);   // v.y is 0 or NaN there
      l = fmaf(f, v.y, l);
      acc.x = fmaf(f, o.x, acc.x);
      acc.y = fmaf(f, o.y, acc.y);
    }
    __syncthreads();   // red is free again
    red[warp][lane] = acc;
    if (lane == 0) red_l[warp] = l;
    __syncthreads();
    if (warp == 0) {
      acc = make_float2(0.f, 0.f);
      l = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        acc.x += red[w][lane].x;
        acc.y += red[w][lane].y;
        l += red_l[w];
      }
      const float inv = l != 0.f ? 1.f / l : 0.f;   // nothing attended: zeros
      reinterpret_cast<uint32_t*>(a.out + ((int64_t)b * a.Hq + hq) * D + sl * K8F_COLS)[lane] =
          pack_bf16x2_rn(acc.x * inv, acc.y * inv);
    }
  }
}

int kv8_box_rows() { return K8_SUB; }

template <int D>
static int launch_t(const CUtensorMap& tmap, const Kv8DecodeArgs& a, cudaStream_t stream) {
  using L = K8Smem<D>;
  const bool weigh = a.w_out != nullptr;
  const void* kernel = weigh ? (const void*)kv8_split_kernel<D, true>
                             : (const void*)kv8_split_kernel<D, false>;
  if (smem_optin(kernel, L::TOTAL) != JF_OK) return JF_ERR_CUDA;
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.budget, (unsigned)a.Hkv);
  cfg.blockDim = dim3(K8_NW * 32);
  cfg.dynamicSmemBytes = L::TOTAL;
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  const cudaError_t e = weigh ? cudaLaunchKernelEx(&cfg, kv8_split_kernel<D, true>, tmap, a)
                              : cudaLaunchKernelEx(&cfg, kv8_split_kernel<D, false>, tmap, a);
  if (e != cudaSuccess) return JF_ERR_CUDA;
  cfg.gridDim = dim3((unsigned)(a.slices * a.Hq * a.B + a.wtiles * a.Hkv * a.B));
  cfg.blockDim = dim3(K8F_THREADS);
  cfg.dynamicSmemBytes = 0;
  const cudaError_t m = weigh ? cudaLaunchKernelEx(&cfg, kv8_merge_kernel<D, true>, a)
                              : cudaLaunchKernelEx(&cfg, kv8_merge_kernel<D, false>, a);
  return m == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

// floats of the scores of one (request, KV head)
int64_t kv8_score_floats(int64_t G, int64_t wstride) {
  return (wstride + K8_SUB - 1) / K8_SUB * 32 * ((G + 1) / 2);
}

// weights (w_out non-null): `scores`, 16-byte aligned, holds the scores of the
// B * Hkv (request, KV head) pairs
int launch_kv8_decode(const Geom& g, const jf_kv_pool& pool, const CUtensorMap& tmap,
                      const int32_t* page_table, int32_t pt_stride, const int32_t* context_lens,
                      int32_t batch, const void* q, int32_t Hq, float softmax_scale, void* out,
                      void* workspace, int32_t num_splits, float* scores, const float* w_in,
                      float* w_out, int64_t wstride, cudaStream_t stream) {
  Kv8DecodeArgs a;
  a.pool = static_cast<const uint8_t*>(pool.base);
  a.num_pages = g.num_pages;
  a.page_bytes = g.page_bytes;
  a.codes_region = g.codes_region;
  a.sb_region = g.sb_region;
  a.P = g.P;
  a.log2P = __builtin_ctz((unsigned)g.P);
  a.Hkv = g.Hkv;
  a.Hq = Hq;
  a.G = Hq / g.Hkv;
  a.B = batch;
  a.page_table = page_table;
  a.pt_stride = pt_stride;
  a.ctx = context_lens;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const int64_t rows = (int64_t)batch * Hq * num_splits;
  a.status = reinterpret_cast<int32_t*>(ws);
  a.part_ml = reinterpret_cast<float*>(ws + 256);
  a.part_o = reinterpret_cast<float*>(ws + 256 + (rows * 8 + 255) / 256 * 256);
  // pieces per KV head: one CTA per SM in all, and B + pieces - 1 partial rows
  // per query row inside the workspace's B * num_splits
  const int slots = sm_count() / g.Hkv > 1 ? sm_count() / g.Hkv : 1;
  const int64_t fit = (int64_t)batch * (num_splits - 1) + 1;
  a.budget = (int)(fit < slots ? fit : slots);
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  a.scores = scores;
  a.w_in = w_in;
  a.w_out = w_out;
  a.wstride = wstride;
  a.pairs = (a.G + 1) / 2;
  a.sstride = kv8_score_floats(a.G, wstride);
  // few query rows: a CTA for each 64 columns; many: one for the row
  const int64_t qrows = (int64_t)batch * Hq;
  a.slices = qrows * (g.D / K8F_COLS) <= 4 * sm_count() ? g.D / K8F_COLS : 1;
  // Weighing CTAs of one, two or four steps: the shortest with which no more than 4 an SM
  // are launched, since each works out its heads' m and l anew (1,024, 2,048 and 4,096
  // positions a CTA: one request of 5,000, 2 KV heads, 8.7, 9.5 and 11.1 us; 16 to 9,000,
  // 4 heads, 21.1, 20.4 and 21.3; 32 to 65,535, 4 heads, 213, 208 and 205).
  int64_t wtiles = 0;
  a.wsteps = 1;
  for (int steps = 1; w_out && steps <= 4; steps *= 2) {
    a.wsteps = steps;
    wtiles = (wstride + (int64_t)steps * K8W_STEP - 1) / ((int64_t)steps * K8W_STEP);
    if (wtiles * batch * g.Hkv <= 4 * sm_count()) break;
  }
  if (qrows * a.slices + wtiles * batch * g.Hkv > 0x7FFFFFFF || g.Hkv > 65535)
    return JF_ERR_UNSUPPORTED;
  a.wtiles = (int)wtiles;
  return g.D == 256 ? launch_t<256>(tmap, a, stream) : launch_t<128>(tmap, a, stream);
}

}  // namespace jfkv
