// Prefill-chunk attention over the latent cache in the expanded form, on the
// 5th-generation tensor cores: the heads' keys and values are worked out from the
// latents once (latent_expand_kernel), then attention runs over them
// (latent_prefill_kernel), as many heads at a time as the workspace holds.
//
// Expansion: [positions, R] times [R, 128 + 128] of a head, M = 256 positions and N =
// 256 channels a CTA pair, CTA 0 supplying the key's weights and CTA 1 the value's;
// the products of a tile run while the tile before goes out.  Positions past the last
// are written as zeros, so that a weight of zero finds no NaN there.  A value of the
// chunk's own positions that is not finite would reach queries before it the same way
// (0 * NaN): it is written as zero and the first such position of each 32 noted, and the
// queries that see it get NaN at the end.
//
// Attention: 256 queries of a head a CTA pair (M = 256, 128 rows each), tiles of 128
// positions of which each CTA supplies 64 keys (128 expanded channels, and the 64
// rotated ones straight from the pool) and 64 of the values' channels.  S is taken
// into three buffers of tensor memory, up to two tiles ahead of P V; P replaces S; O
// stays in tensor memory.  Two groups of four softmax warps take the even and the odd
// tiles, a row a thread; the group with an item's last tile takes O out, while the other
// is at the next item's first.  Keys and queries multiply as bf16; values and weights as
// fp16, whose three more bits they need: in bf16 the two roundings weighed as much as the
// output's own (a whole prompt of 4,095 off by 0.0026 of its norm for the 0.0017 of
// rounding exact values).  fp16's range is not bf16's, so a head's values of a tile of 128
// positions are held as v 2^-e, e a whole number that puts the largest between 2^14 and 2^15, and a
// position counts by s + e: its weight is 2^(s + e - m), and O = sum of weight times held
// value is in units of 2^m whatever e.  A row's reference m is a whole number too (powers of
// two change no other bits), set so that the largest weight is about 2^10; it moves, O's row
// with it, when a weight passes 2^15.9.  The sum of 2^s has a reference of its own: each tile's weights
// add 2^(m - e) times theirs, and what is stored as nothing beside far larger values still counts.
// A value's error is 2^-11 of it, or 2^-39 of its tile's largest.  (In fp16 as they are, values of
// 2^-20 gave outputs off by 0.017 of their norm, of 2^-30 zeros.)
//
// What bounds it: the tensor cores at the power they may take.  2,048 queries after 30,720
// positions x 16 heads take 467 to 487 us; each kernel alone: expansion 81 (137 GFLOP, 1,690 TFLOP/s, the
// tensor pipe 73 % active), attention 392 (667 GFLOP, 1,700 TFLOP/s, 91 %), the join 9.  Expanding costs 2 R
// 256 operations a position and head once and saves 1,536 of 2,176 a (query, position) pair of the
// absorbed form: from about 170 queries on it is less.  Below that (77 queries after 4,001 x 16
// heads: 32.7 us, with their launches expansion 15, attention 13, join 5) the absorbed form's products would be 6 us
// against 11, but it would need two products with the weights around the decode and its join.
//
// Work: the (head, 256 queries) items' tiles, and a header each, are laid end to end and
// cut into one run of equal length per pair; a cut item's parts are joined by
// latent_prefill_merge_kernel.
#include <cmath>

#include "latent_tc.cuh"

namespace jfkv {

constexpr int LP_T = 128;            // positions a tile
constexpr int LP_Q = 256;            // queries a pair
constexpr int LP_HDR = 2;            // an item's fixed cost, in tiles
constexpr float LP_SET = 10.f;       // a reference puts the largest weight at 2^9.5 to 2^10.5;
// it moves when one passes 2^15.9 (fp16 ends below 2^16).  With floor() and 15, powers that differ by one
// between tiles made it move more often: 2,048 queries after 30,720 positions 486 us for 475.
constexpr float LP_TOP = 15.9f;
constexpr float LP_FAR = 100.f;      // weights this far below 2^s (log2) are not summed as stored
constexpr int LP_NONE = 0x7FFFFFFF;  // no position

struct LatentChunk {                 // one pass: heads h0 .. h0 + heads - 1
  LatentPool pool;
  const int32_t* pt;
  uint16_t* k;                       // [heads][n_pad][128] bf16
  uint16_t* v;                       // the same, fp16
  uint16_t* out;                     // [C][H][128]
  int32_t* bad;                      // [heads][n_pad / 32]: first position of a value that is not finite
  float* power;                      // [heads][n_pad / 128]: e of a tile, -infinity where all its values are zero
  int32_t* status;
  float4* ml;                        // [2 * pairs * 256]: O's reference, the sum's, the sum, -
  float* o;                          // [2 * pairs * 256][128]
  int64_t units, units_head;         // of the pass, of a head
  int32_t n, n_pad, q_start, C, H, h0, heads, causal;
  int32_t q_tiles, pairs;
  uint32_t inv;                      // of the pairs, for PairRuns
  float scale_log2;
};

// ===========================================================================
// Expansion
// ===========================================================================
// A pair takes a run of (256 positions, head) tiles, heads within positions, and keeps the
// positions' latents in shared memory while the heads' weights stream past: with both
// streamed a CTA read 64 bytes a cycle, more than the L2 cache gives all of them (2,048 queries
// after 30,720 positions x 16 heads 525 us, 501 so).
constexpr int LE_STAGES = 4;
constexpr int LE_CHUNKS = 8;           // 64-channel chunks of R at most
constexpr int LE_THREADS = 32 * 12;
struct LeSmem {
  static constexpr int CHUNK = 128 * 128;                          // 64 channels of 128 rows
  static constexpr int OFF_B = LE_CHUNKS * CHUNK;
  static constexpr int OFF_OUT = OFF_B + LE_STAGES * CHUNK;        // 8 warps x [32 rows][128 B]
  static constexpr int OFF_BAR = OFF_OUT + 8 * 4096;
  static constexpr int OFF_TOP = OFF_BAR + 512;                    // [2][4] largest magnitudes, tile t % 2
  static constexpr int TOTAL = OFF_TOP + 32;
  static_assert(TOTAL <= 227 * 1024, "shared memory per CTA");
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LE_THREADS, 1)
latent_expand_kernel(const __grid_constant__ CUtensorMap pmap, const __grid_constant__ CUtensorMap kmap,
                     const __grid_constant__ CUtensorMap vmap, const __grid_constant__ LatentChunk a) {
  using L = LeSmem;
  constexpr uint32_t ID = idesc_bf16(256, 256, 0);
  extern __shared__ __align__(1024) uint8_t sm[];
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sm + L::OFF_BAR);
  uint64_t* const b_full = bars + 0;    // [4] on CTA 0: both CTAs' weights of a stage
  uint64_t* const a_full = bars + 4;    // [8] on CTA 0: both CTAs' latents, 64 channels
  uint64_t* const b_land = bars + 12;   // [4] CTA 1's
  uint64_t* const a_land = bars + 16;   // [8]
  uint64_t* const b_free = bars + 24;   // [4] stage read
  uint64_t* const a_free = bars + 28;   // all products with these latents done
  uint64_t* const d_full = bars + 29;   // [2] a tile's products done
  uint64_t* const d_free = bars + 31;   // [2] on CTA 0: and gone out, in both CTAs
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 33);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);   // uniform
  const int lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (warp == 0) {
    tc::alloc2(tmem_slot, 512);
  } else if (warp == 1) {   // a barrier a thread
    if (lane == 0) prefetch_tensormap(&pmap);
    if (lane == 1) prefetch_tensormap(rank ? &vmap : &kmap);
    // b_full, a_full: both CTAs; d_free: their 16 warps; the others one arrival
    mbar_init(&bars[lane], lane < 12 ? 2 : lane >= 31 ? 16 : 1);
    if (lane == 0) mbar_init(&bars[32], 16);
    fence_barrier_init();
  }
  // tiles of a pass: below 2^24, and their product with the pairs below 2^31
  const uint32_t tiles = (uint32_t)(a.n_pad / 256) * (uint32_t)a.heads;
  const uint32_t i0 = tiles * pair / pairs, i1 = tiles * (pair + 1) / pairs;
  int pt = (int)(i0 / a.heads), hl = (int)(i0 - pt * a.heads);   // of the current tile
  const bool placed = !(smem_u32(sm) & 1023u);   // the swizzled layouts need it; the same in both CTAs
  const int count = placed ? (int)(i1 - i0) : 0, steps = a.pool.R / 64;
  tc::fence_before();
  __syncthreads();
  tc::cluster_sync();   // both CTAs: barriers initialized, TMEM allocated
  tc::fence_after();
  auto advance = [&] {
    if (++hl == a.heads) {
      hl = 0;
      ++pt;
    }
  };
  asm volatile("griddepcontrol.wait;\n" ::: "memory");   // what came before has been written
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  if (!placed && threadIdx.x == 0) flag_error(a.status, JF_DEV_ERR_LAYOUT);

  bool ok = true;
  if (warp == 0) {
    int st = 0, ph = 0, na = 0;   // stage, how often the ring went round, latents taken so far
    if (rank == 0) {
      const uint32_t leader = elect_one();
      const uint64_t ad = tc::sdesc_sw128(smem_u32(sm), 16, 1024);
      const uint64_t bd = tc::sdesc_sw128(smem_u32(sm + L::OFF_B), 16, 1024);
      auto wait = [&](uint64_t* bar, int phase) {
        return __all_sync(0xffffffffu, mbar_wait_bounded(bar, phase & 1)) != 0;
      };
      for (int t = 0; t < count && ok; ++t) {
        const bool fresh = t == 0 || hl == 0;
        if (t >= 2) ok = wait(&d_free[t & 1], (t >> 1) - 1);
        tc::fence_after();
        const uint32_t d = (t & 1) * 256;
        for (int s = 0; s < steps && ok; ++s) {
          if (fresh) ok = wait(&a_full[s], na);
          ok = ok && wait(&b_full[st], ph);
          tc::fence_after();
          const uint64_t at = ad + (uint64_t)(s * (L::CHUNK >> 4)), bt = bd + (uint64_t)(st * (L::CHUNK >> 4));
          if (ok) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma2_ss_if(leader, d, at + ((k * 32) >> 4), bt + ((k * 32) >> 4), ID,
                         (s > 0 || k > 0) ? 1u : 0u);
            if (t * steps + s < count * steps - LE_STAGES) tc::commit2_both_if(leader, &b_free[st]);   // waited for
          }
          if (++st == LE_STAGES) {
            st = 0;
            ++ph;
          }
        }
        if (fresh) ++na;
        advance();
        if (ok && hl == 0 && t + 1 < count) tc::commit2_both_if(leader, a_free);   // waited for
        if (ok) tc::commit2_both_if(leader, &d_full[t & 1]);
      }
      for (int t = max(0, count - 2); t < count && ok; ++t) ok = wait(&d_free[t & 1], t >> 1);
    } else if (lane == 0) {
      for (int t = 0; t < count && ok; ++t) {
        const bool fresh = t == 0 || hl == 0;
        for (int s = 0; s < steps && ok; ++s) {
          if (fresh) {
            ok = mbar_wait_bounded(&a_land[s], na & 1);
            if (ok) tc::arrive_cluster(&a_full[s], 0);
          }
          if (ok) ok = mbar_wait_bounded(&b_land[st], ph & 1);
          if (ok) tc::arrive_cluster(&b_full[st], 0);
          if (++st == LE_STAGES) {
            st = 0;
            ++ph;
          }
        }
        if (fresh) ++na;
        advance();
      }
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    __syncwarp();
  } else if (warp == 1) {
    // ---- weights: the keys' 128 rows of the head (CTA 0), the values' (CTA 1) ----------------
    if (lane == 0) {
      int st = 0, ph = 0;
      for (int t = 0; t < count && ok; ++t, advance())
        for (int s = 0; s < steps; ++s) {
          if (ph > 0 && !mbar_wait_bounded(&b_free[st], (ph - 1) & 1)) {
            ok = false;
            break;
          }
          uint64_t* const bar = rank == 0 ? &b_full[st] : &b_land[st];
          mbar_arrive_expect_tx(bar, L::CHUNK);
          tma_load_2d(smem_u32(sm + L::OFF_B + st * L::CHUNK), rank ? &vmap : &kmap, s * 64,
                      (a.h0 + hl) * 128, bar);
          if (++st == LE_STAGES) {
            st = 0;
            ++ph;
          }
        }
      if (!ok) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---- latents: this CTA's 128 of the 256 positions -----------------------------------
    if (lane == 0) {
      int na = 0;
      for (int t = 0; t < count && ok; ++t, advance()) {
        if (t > 0 && hl > 0) continue;
        if (na > 0 && !mbar_wait_bounded(a_free, (na - 1) & 1)) {
          ok = false;
          break;
        }
        ++na;
        const int pos = pt * 256 + 128 * (int)rank;
        const int row0 = half_row(a.pool, a.pt, pos, a.n, a.status);
        const int row1 = half_row(a.pool, a.pt, pos + 64, a.n, a.status);
        for (int s = 0; s < steps; ++s) {
          uint64_t* const bar = rank == 0 ? &a_full[s] : &a_land[s];
          mbar_arrive_expect_tx(bar, L::CHUNK);
          const uint32_t dst = smem_u32(sm) + s * L::CHUNK;
          tma_load_2d(dst, &pmap, s * 64, row0, bar);
          tma_load_2d(dst + 8192, &pmap, s * 64, row1, bar);
        }
      }
      if (!ok) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ---- out: warps 4-7 the keys' 128 columns, 8-11 the values' -----------------------
    const int quarter = warp & 3, kind = warp >= 8 ? 1 : 0;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t tr = smem_u32(sm + L::OFF_OUT) + (warp - 4) * 4096;
    uint16_t* const dst = kind ? a.v : a.k;
    uint32_t* const s_top = reinterpret_cast<uint32_t*>(sm + L::OFF_TOP);
    // values of positions that not every query of the chunk sees
    const int apart = kind && a.causal ? a.q_start + 1 : LP_NONE;
    for (int t = 0; t < count; ++t, advance()) {
      const int pos0 = pt * 256 + 128 * (int)rank + quarter * 32;
      const int pos = pos0 + lane;
      // A wait that gave up ends the work but not the meetings: the four warps of a tile's values would wait
      // for one another for ever.
      ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&d_full[t & 1], (t >> 1) & 1)) != 0;
      tc::fence_after();
      int first = LP_NONE;
      float power = -INFINITY, scale = 1.f;
      if (kind) {
        // The largest finite magnitude of the tile, as twice its bits and 2^24: those of infinities and NaN
        // pass 2^32 and come out below 2^24.
        uint32_t top = 0u;
        if (ok) {
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            uint32_t x[32];
            tc::ld32((t & 1) * 256 + 128 + c0 + lane_off, x);
            tc::wait_ld();
#pragma unroll
            for (int c = 0; c < 32; ++c) top = max(top, 2u * x[c] + (1u << 24));
          }
        }
        top = __reduce_max_sync(0xffffffffu, pos < a.n ? top : 0u);
        if (lane == 0) s_top[4 * (t & 1) + quarter] = top;
        // two buffers: a warp may be at the next tile before the others have read this one's
        asm volatile("bar.sync 1, 128;\n" ::: "memory");
        const uint4 of = lds128(smem_u32(s_top + 4 * (t & 1)));
        top = max(max(of.x, of.y), max(of.z, of.w));
        if (top > 1u << 24) {   // to between 2^14 and 2^15; by 2^126 at most, from 2^-112 down
          const int expo = max((int)(top >> 24) - 1, 15);
          power = (float)(expo - 141);
          scale = __uint_as_float((uint32_t)(268 - expo) << 23);
          if (top >= 2u * 0x477FF000u + (1u << 24) && lane == 0)   // 65,520: past fp16 as it is
            flag_error(a.status, JF_DEV_ERR_RANGE);
        }
      }
      if (!ok) continue;
#pragma unroll 1
      for (int c0 = 0; c0 < 128; c0 += 64) {
        uint32_t x[2][32];
        tc::ld32((t & 1) * 256 + kind * 128 + c0 + lane_off, x[0]);
        tc::ld32((t & 1) * 256 + kind * 128 + c0 + 32 + lane_off, x[1]);
        tc::wait_ld();
        if (c0 == 64) {   // the tile's columns have been read
          tc::fence_before();
          __syncwarp();
          if (lane == 0) tc::arrive_cluster(&d_free[t & 1], 0);
        }
        uint32_t w[32], top = 0u;   // the values, and the largest magnitudes' bits of both halves
        if (kind) {
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            w[c] = pack_f16x2(__uint_as_float(x[c >> 4][(2 * c) & 31]) * scale,
                              __uint_as_float(x[c >> 4][(2 * c + 1) & 31]) * scale);
            top = __vmaxu2(top, w[c] & 0x7FFF7FFFu);
          }
        } else {
#pragma unroll
          for (int c = 0; c < 32; ++c)
            w[c] = pack_bf16x2(__uint_as_float(x[c >> 4][(2 * c) & 31]), __uint_as_float(x[c >> 4][(2 * c + 1) & 31]));
        }
        if (pos0 + 31 >= a.n) {   // positions past the last
#pragma unroll
          for (int c = 0; c < 32; ++c)
            if (pos >= a.n) w[c] = 0u;
          if (pos >= a.n) top = 0u;
        }
        if (pos >= apart && max(top & 0xFFFFu, top >> 16) >= 0x7C00u) {   // a value that is not finite
          first = pos;
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            if ((w[c] & 0x7C00u) == 0x7C00u) w[c] &= 0xFFFF0000u;
            if ((w[c] & 0x7C000000u) == 0x7C000000u) w[c] &= 0xFFFFu;
          }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sts128(tr + lane * 128 + ((k ^ (lane & 7)) << 4), w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        __syncwarp();
        uint16_t* const to = dst + ((int64_t)hl * a.n_pad + pos0) * 128 + c0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int row = u * 4 + (lane >> 3), piece = lane & 7;
          *reinterpret_cast<uint4*>(to + row * 128 + piece * 8) =
              lds128(tr + row * 128 + ((piece ^ (row & 7)) << 4));
        }
        __syncwarp();
      }
      if (kind) {
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) {
          const int64_t at = (int64_t)hl * a.n_pad + pos0;
          a.bad[at >> 5] = first;
          if (quarter == 0) a.power[at >> 7] = power;
        }
      }
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
  }
  // Neither CTA may release TMEM or exit while its partner can still reach it.  CTA 1's arrivals were all waited
  // for, the last ones at the issuer's end, the products' at d_full on the way out, at b_free and a_free by the
  // next copies: where none is to come, no arrival is asked for.
  tc::fence_before();
  settle(ok);
  cluster_meet();
  if (warp == 0) {
    tc::fence_after();
    tc::dealloc2(*tmem_slot, 512);
  }
}

// ===========================================================================
// Attention
// ===========================================================================
constexpr int LA_THREADS = 32 * 12;
constexpr int LA_KS = 3, LA_VS = 4, LA_SB = 3;   // LA_VS: also of pv_done
struct LaSmem {
  static constexpr int Q_BYTES = 3 * 128 * 128;         // [64-channel chunk][128 rows][128 B]
  static constexpr int K_BYTES = 3 * 64 * 128;          // [64-channel chunk][64 positions][128 B]
  static constexpr int V_BYTES = 128 * 128;             // 64 channels of 128 positions
  static constexpr int OFF_K = Q_BYTES;
  static constexpr int OFF_V = OFF_K + LA_KS * K_BYTES;
  static constexpr int OFF_OUT = OFF_V + LA_VS * V_BYTES;   // 8 warps x [32 rows][128 B]
  static constexpr int OFF_BAR = OFF_OUT + 8 * 4096;
  static constexpr int OFF_M = OFF_BAR + 512;           // [4][128] O's references after tile t % 4
  static constexpr int OFF_L = OFF_M + 4 * 128 * 4;     // [4][128] (reference, sum) of segment s % 4, from one group to the other
  static constexpr int TOTAL = OFF_L + 4 * 128 * 8;
  static_assert(TOTAL <= 227 * 1024, "shared memory per CTA");
};

// 2^(m - ms), the unit of O over that of the sum, in two factors: one alone could leave fp32's range where the
// output does not
__device__ __forceinline__ float half_power(float m, float ms, float* rest) {
  const float k = m == -INFINITY || ms == -INFINITY ? 0.f : m - ms, half = floorf(0.5f * k);
  *rest = fast_exp2(k - half);
  return fast_exp2(half);
}

// tiles and first unit (of its head) of query tile qt
__device__ __forceinline__ int chunk_tiles(const LatentChunk& a, int qt) {
  if (!a.causal) return (a.n + LP_T - 1) / LP_T;
  const int64_t seen = (int64_t)a.q_start + (int64_t)(qt + 1) * LP_Q;
  return (int)(((seen < a.n ? seen : a.n) + LP_T - 1) / LP_T);
}
__device__ __forceinline__ int64_t chunk_start(const LatentChunk& a, int qt) {
  const int64_t q = qt;
  if (!a.causal) return q * ((a.n + LP_T - 1) / LP_T + LP_HDR);
  // tiles before the last query tile: 2 (qt + 1) + ceil(q_start / 128)
  return q * (q - 1) + q * (2 + (a.q_start + LP_T - 1) / LP_T + LP_HDR);
}

struct ChunkSeg {
  int hl, qt, j0, j1, n;
};
struct ChunkIter {
  int64_t start, u0, u1;   // first unit of item (hl, qt); the pair's run
  int hl, qt;
};

__device__ __forceinline__ ChunkIter chunk_run(const LatentChunk& a, int pair) {
  const PairRuns runs(a.units, a.pairs, a.inv);
  ChunkIter s;
  s.u0 = runs.first(pair);
  s.u1 = runs.first(pair + 1);
  s.hl = (int)divide((uint64_t)s.u0, (uint64_t)a.units_head);
  const int64_t in = s.u0 - s.hl * a.units_head;
  int lo = 0, hi = a.q_tiles - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (chunk_start(a, mid) <= in) lo = mid; else hi = mid - 1;
  }
  s.qt = lo;
  s.start = s.hl * a.units_head + chunk_start(a, lo);
  return s;
}
__device__ __forceinline__ bool next_chunk_seg(const LatentChunk& a, ChunkIter& s, ChunkSeg& g) {
  while (s.start < s.u1 && s.hl < a.heads) {
    const int n = chunk_tiles(a, s.qt);
    const int64_t first = s.start + LP_HDR;
    const int64_t lo = max((int64_t)0, s.u0 - first), hi = min((int64_t)n, s.u1 - first);
    g.hl = s.hl;
    g.qt = s.qt;
    g.n = n;
    s.start += n + LP_HDR;
    if (++s.qt == a.q_tiles) {
      s.qt = 0;
      ++s.hl;
    }
    if (lo < hi) {
      g.j0 = (int)lo;
      g.j1 = (int)hi;
      return true;
    }
  }
  return false;
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LA_THREADS, 1)
latent_prefill_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap pmap,
                      const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                      const __grid_constant__ LatentChunk a) {
  using L = LaSmem;
  constexpr uint32_t IDQK = idesc_bf16(256, LP_T, 0);
  constexpr uint32_t IDPV = tc::idesc_f16_f32(256, 128, 0, 1);
  extern __shared__ __align__(1024) uint8_t sm[];
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sm + L::OFF_BAR);
  // on CTA 0, where the pair's MMAs are issued:
  uint64_t* const k_full = bars + 0;     // [3] both CTAs' K of a tile
  uint64_t* const v_full = bars + 3;     // [4] both CTAs' V
  uint64_t* const q_full = bars + 7;     // both CTAs' Q of a segment
  uint64_t* const p_ready = bars + 8;    // [4] both CTAs' P of tile t % 4
  // on each CTA:
  uint64_t* const k_land = bars + 12;    // [3] CTA 1: its operands have landed
  uint64_t* const v_land = bars + 15;    // [4]
  uint64_t* const q_land = bars + 19;
  uint64_t* const k_free = bars + 20;    // [3] stage read
  uint64_t* const pv_done = bars + 23;   // [4] P V of tile t % 4, and so V's stage read
  uint64_t* const q_free = bars + 27;    // products with a segment's Q done
  uint64_t* const s_full = bars + 28;    // [3] S of tile t % 3
  // [4][4 quarters] the reference after tile t % 4 is set.  (One barrier a group would do but for a
  // group that takes O out: the other may be two of its tiles on, and a parity then says no for ever.)
  uint64_t* const m_bar = bars + 35;
  uint64_t* const o_free = bars + 51;    // on CTA 0: both CTAs have read a segment's O
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 52);
  float* const s_m = reinterpret_cast<float*>(sm + L::OFF_M);
  float2* const s_ml = reinterpret_cast<float2*>(sm + L::OFF_L);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);   // uniform
  const int lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  const int pair = (int)(blockIdx.x >> 1);
  if (warp == 0) {
    tc::alloc2(tmem_slot, 512);
  } else if (warp == 1) {   // a barrier a thread
    if (lane == 0) prefetch_tensormap(&qmap);
    if (lane == 1) prefetch_tensormap(&pmap);
    if (lane == 2) prefetch_tensormap(&kmap);
    if (lane == 3) prefetch_tensormap(&vmap);
    // k_full, v_full, q_full: both CTAs; p_ready, o_free: their eight warps; the others one arrival
    mbar_init(&bars[lane], lane < 8 ? 2 : lane < 12 ? 8 : 1);
    if (lane < 20) mbar_init(&bars[32 + lane], lane == 19 ? 8 : 1);
    fence_barrier_init();
  }
  // the first segment, in one copy of that code for all roles: it is fetched when it first runs
  ChunkIter run = chunk_run(a, pair);
  ChunkSeg sg;
  const bool placed = !(smem_u32(sm) & 1023u);   // the swizzled layouts need it; the same in both CTAs
  if (!placed) run.hl = a.heads;                 // no work
  bool more = next_chunk_seg(a, run, sg);
  tc::fence_before();
  __syncthreads();
  tc::cluster_sync();   // both CTAs: barriers initialized, TMEM allocated
  tc::fence_after();
  asm volatile("griddepcontrol.wait;\n" ::: "memory");   // the keys and values have been written
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  if (!placed && threadIdx.x == 0) flag_error(a.status, JF_DEV_ERR_LAYOUT);
  // all 512 columns are this CTA's: O from 0, the S buffers behind it
  constexpr uint32_t tO = 0, tS = 128;

  bool ok = true;
  if (warp == 0) {
    if (rank == 0) {
      // ================= MMA issuer (the whole warp: control flow stays uniform) ==========
      const uint32_t leader = elect_one();
      const uint64_t qd = tc::sdesc_sw128(smem_u32(sm), 16, 1024);
      const uint64_t kd = tc::sdesc_sw128(smem_u32(sm + L::OFF_K), 16, 1024);
      const uint64_t vd = tc::sdesc_sw128(smem_u32(sm + L::OFF_V), 16, 1024);
      // S of tile qi (of qleft more of its segment) up to two tiles before P V of tile pi, across the
      // segments' ends; but a segment's last P V go first as soon as they can, since O's way out waits
      // for them.
      auto wait = [&](uint64_t* bar, int phase) {
        return __all_sync(0xffffffffu, mbar_wait_bounded(bar, phase & 1)) != 0;
      };
      ChunkIter prun = run;
      const int first = __shfl_sync(0xffffffffu, more ? sg.j1 - sg.j0 : 0, 0);
      int qi = 0, qleft = first, qseg = 0, pi = 0, pleft = 0, pseg = 0;
      bool fresh_q = true, fresh_o = false;   // the segment's first S, its first P V
      while (ok) {
        if (qleft == 0 && more) {
          more = __all_sync(0xffffffffu, next_chunk_seg(a, run, sg)) != 0;
          qleft = more ? __shfl_sync(0xffffffffu, sg.j1 - sg.j0, 0) : 0;
          fresh_q = true;
        }
        const bool last_pv = pi < qi && (fresh_q || qseg > pseg) && pleft > 0;   // S is a segment ahead
        if (qleft > 0 && qi - pi < LA_SB &&
            (!last_pv || (!__all_sync(0xffffffffu, mbar_test(&p_ready[pi & 3], pi >> 2)) &&
                          (!fresh_q || __all_sync(0xffffffffu, mbar_test(q_full, qseg)))))) {
          const int st = qi % LA_KS;
          if (fresh_q) ok = wait(q_full, qseg++);
          ok = ok && wait(&k_full[st], qi / LA_KS);
          tc::fence_after();
          const uint64_t k0 = kd + (uint64_t)(st * (L::K_BYTES >> 4));
          const uint32_t d = tS + (qi % LA_SB) * 128;
          fresh_q = false;
          ++qi;
          --qleft;
          if (ok) {
#pragma unroll
            for (int k = 0; k < 12; ++k)
              mma2_ss_if(leader, d, qd + (((k >> 2) * 128 * 128 + (k & 3) * 32) >> 4),
                         k0 + (((k >> 2) * 64 * 128 + (k & 3) * 32) >> 4), IDQK, k > 0 ? 1u : 0u);
            tc::commit2_both_if(leader, &k_free[st]);
            tc::commit2_both_if(leader, &s_full[(qi - 1) % LA_SB]);
            if (qleft == 0) tc::commit2_both_if(leader, q_free);
          }
        } else if (pi < qi) {
          if (pleft == 0) {
            pleft = first;
            if (pseg > 0) {
              next_chunk_seg(a, prun, sg);
              pleft = __shfl_sync(0xffffffffu, sg.j1 - sg.j0, 0);
              ok = wait(o_free, pseg - 1);
            }
            fresh_o = true;
            ++pseg;
          }
          const int st = pi % LA_VS;
          ok = ok && wait(&p_ready[pi & 3], pi >> 2) && wait(&v_full[st], pi / LA_VS);
          tc::fence_after();
          const uint64_t v0 = vd + (uint64_t)(st * (L::V_BYTES >> 4));
          const uint32_t p = tS + (pi % LA_SB) * 128;
          if (ok) {
#pragma unroll
            for (int k = 0; k < LP_T / 16; ++k)
              tc::mma2_ts_if(leader, tO, p + 8 * k, v0 + ((k * 2048) >> 4), IDPV,
                             (!fresh_o || k > 0) ? 1u : 0u);
            tc::commit2_both_if(leader, &pv_done[pi & 3]);
          }
          fresh_o = false;
          ++pi;
          --pleft;
        } else {
          break;   // nothing left
        }
      }
      if (ok && pseg > 0) ok = wait(o_free, pseg - 1);
    } else if (lane == 0) {
      // ================= CTA 1's arrivals =================
      int t = 0;
      auto pass_v = [&](int T) {
        ok = mbar_wait_bounded(&v_land[T % LA_VS], (T / LA_VS) & 1);
        if (ok) tc::arrive_cluster(&v_full[T % LA_VS], 0);
      };
      for (; ok && more; more = next_chunk_seg(a, run, sg))
        for (int j = sg.j0; j < sg.j1 && ok; ++j, ++t) {
          ok = mbar_wait_bounded(&k_land[t % LA_KS], (t / LA_KS) & 1);
          if (ok) tc::arrive_cluster(&k_full[t % LA_KS], 0);
          if (ok && t >= 2) pass_v(t - 2);
        }
      for (int T = max(0, t - 2); T < t && ok; ++T) pass_v(T);
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    __syncwarp();
  } else if (warp == 1) {
    // ================= K: this CTA's 64 positions of each tile =================
    if (lane == 0) {
      int t = 0;
      for (;; more = next_chunk_seg(a, run, sg)) {
        // after the last segment a turn over the ring that waits and brings nothing: each stage's last products
        // have told both CTAs before either ends
        const int j0 = more ? sg.j0 : 0, j1 = more ? sg.j1 : LA_KS;
        int y = more ? half_row(a.pool, a.pt, j0 * LP_T + 64 * (int)rank, a.n, a.status) : 0;
        for (int j = j0; j < j1; ++j, ++t) {
          const int row = y, st = t % LA_KS, pos = j * LP_T + 64 * (int)rank;
          if (more && j + 1 < j1) y = half_row(a.pool, a.pt, pos + LP_T, a.n, a.status);
          if (t >= LA_KS && !mbar_wait_bounded(&k_free[st], (t / LA_KS - 1) & 1)) {
            ok = false;
            break;
          }
          if (!more) continue;
          uint64_t* const land = rank == 0 ? &k_full[st] : &k_land[st];
          mbar_arrive_expect_tx(land, L::K_BYTES);
          const uint32_t dst = smem_u32(sm + L::OFF_K + st * L::K_BYTES);
          const int at = sg.hl * a.n_pad + pos;
          tma_load_2d(dst, &kmap, 0, at, land);
          tma_load_2d(dst + 8192, &kmap, 64, at, land);
          tma_load_2d(dst + 16384, &pmap, a.pool.R, row, land);
        }
        if (!more || !ok) break;
      }
      if (!ok) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
    __syncwarp();
  } else if (warp == 2) {
    // ================= V: this CTA's 64 channels of all 128 positions =================
    if (lane == 0) {
      int t = 0;
      for (;; more = next_chunk_seg(a, run, sg)) {
        const int j0 = more ? sg.j0 : 0, j1 = more ? sg.j1 : LA_VS;   // a last turn, as K's
        for (int j = j0; j < j1; ++j, ++t) {
          const int st = t % LA_VS;
          if (t >= LA_VS && !mbar_wait_bounded(&pv_done[st], (t / LA_VS - 1) & 1)) {
            ok = false;
            break;
          }
          if (!more) continue;
          uint64_t* const land = rank == 0 ? &v_full[st] : &v_land[st];
          mbar_arrive_expect_tx(land, L::V_BYTES);
          tma_load_2d(smem_u32(sm + L::OFF_V + st * L::V_BYTES), &vmap, 64 * (int)rank,
                      sg.hl * a.n_pad + j * LP_T, land);
        }
        if (!more || !ok) break;
      }
      if (!ok) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
    __syncwarp();
  } else if (warp == 3) {
    // ================= Q: 128 rows; zeros past the chunk's end =================
    if (lane == 0) {
      int nseg = 0;
      for (; ok; more = next_chunk_seg(a, run, sg)) {
        if (nseg > 0 && !mbar_wait_bounded(q_free, (nseg - 1) & 1)) {
          ok = false;
          break;
        }
        if (!more) break;
        ++nseg;
        uint64_t* const land = rank == 0 ? q_full : q_land;
        mbar_arrive_expect_tx(land, L::Q_BYTES);
        for (int c = 0; c < 3; ++c)
          tma_load_3d(smem_u32(sm) + c * 128 * 128, &qmap, c * 64, a.h0 + sg.hl,
                      sg.qt * LP_Q + 128 * (int)rank, land);
        if (rank == 1) {   // passed on to CTA 0
          ok = mbar_wait_bounded(q_land, (nseg - 1) & 1);
          if (ok) tc::arrive_cluster(q_full, 0);
        }
      }
      if (!ok) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
    }
    __syncwarp();
  } else {
    // ================= softmax: group 0 the even tiles, group 1 the odd; O out =================
    const int quarter = warp & 3, group = warp >= 8 ? 1 : 0;
    const int r = quarter * 32 + lane;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const float sc = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
    const uint64_t kk = f32x2(sc, sc);
    int t0 = 0, seg = 0;   // tiles and number of the segments before
    // A wait that gave up ends the work but not the meetings: the other group would wait for ever.
    for (; more; more = next_chunk_seg(a, run, sg), ++seg) {
      const int row0 = sg.qt * LP_Q + 128 * (int)rank + quarter * 32;   // the warp's first query
      auto limit_of = [&](int q) { return a.causal ? min(a.q_start + q, a.n - 1) : a.n - 1; };
      const int limit = limit_of(row0 + lane);         // last position seen
      const int first_limit = limit_of(row0);          // by every query of the warp
      const int nt = sg.j1 - sg.j0;
      const float* const powers = a.power + (((int64_t)sg.hl * a.n_pad) >> 7) + sg.j0;
      float e_next = 0.f;
      if (((t0 + group) & 1) < nt) e_next = powers[(t0 + group) & 1];
      int first_bad = LP_NONE;   // of the values that the warp's queries see and not all of the chunk's
      if (a.causal)
        for (int b = ((a.q_start + 1) >> 5) + lane; b <= (limit_of(row0 + 31) >> 5); b += 32)
          first_bad = min(first_bad, a.bad[(((int64_t)sg.hl * a.n_pad) >> 5) + b]);
      float m_own = -INFINITY;              // O's reference at this group's last tile
      float m_sum = -INFINITY, l = 0.f;     // the group's sum of weights, and its reference
      for (int i = (t0 + group) & 1; i < nt && ok; i += 2) {
        const int T = t0 + i, key0 = (sg.j0 + i) * LP_T;
        const uint32_t tb = tS + (T % LA_SB) * 128 + lane_off;
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(&s_full[T % LA_SB], (T / LA_SB) & 1)) != 0;
        if (!ok) break;
        tc::fence_after();
        // The row's largest score, then the weights: two short loops, each one copy of its code (written
        // out over the 128 positions, the code came from beyond the instruction caches at every tile).
        // What the first changes of S -- the sign of a scale below zero, a scale of zero, positions not
        // seen -- it writes back.
        uint32_t s[2][32];
        const float e = e_next;   // the power that the tile's values are held by
        float x[2] = {-INFINITY, -INFINITY};
        const bool plain = a.scale_log2 > 0.f && key0 + LP_T - 1 <= first_limit;   // of the whole warp
#pragma unroll 1
        for (int c0 = 0; c0 < LP_T; c0 += 64) {
          tc::ld32(tb + c0, s[0]);
          tc::ld32(tb + c0 + 32, s[1]);
          tc::wait_ld();
          if (!plain) {
            if (!(a.scale_log2 > 0.f)) {   // of a scale below zero the sign, of one of zero nothing (or NaN)
#pragma unroll
              for (int c = 0; c < 64; ++c) {
                const uint32_t w = s[c >> 5][c & 31];
                s[c >> 5][c & 31] = a.scale_log2 < 0.f ? w ^ 0x80000000u : __float_as_uint(__uint_as_float(w) * 0.f);
              }
            }
            const int seen = limit - key0 - c0;
#pragma unroll
            for (int c = 0; c < 64; ++c)
              if (c > seen) s[c >> 5][c & 31] = 0xFF800000u;
            tc::st32(tb + c0, s[0]);
            tc::st32(tb + c0 + 32, s[1]);
            tc::wait_st();
          }
#pragma unroll
          for (int c = 0; c < 32; ++c)
            x[c & 1] = max3(x[c & 1], __uint_as_float(s[c >> 4][(2 * c) & 31]),
                            __uint_as_float(s[c >> 4][(2 * c + 1) & 31]));
        }
        const float top = fmaxf(x[0], x[1]), top_e = fmaf(sc, top, e);
        const float mt = sc * top;
        if (mt > m_sum + LP_TOP || m_sum == -INFINITY) {
          const float to = floorf(mt);
          if (m_sum != -INFINITY) l *= fast_exp2(m_sum - to);
          m_sum = to;
        }
        // the reference after the tile before, the other group's
        float m_ref = -INFINITY;   // nothing seen so far
        if (i > 0) {
          ok = __all_sync(0xffffffffu, mbar_wait_bounded(&m_bar[((T - 1) & 3) * 4 + quarter],
                                                         ((T - 1) >> 2) & 1)) != 0;
          if (!ok) break;
          m_ref = s_m[((T - 1) & 3) * 128 + r];
        }
        const float m_new = top_e > m_ref + LP_TOP || m_ref == -INFINITY ? rintf(top_e) - LP_SET : m_ref;
        const bool moves = m_ref != -INFINITY && m_new != m_ref;
        if (__any_sync(0xffffffffu, moves)) {   // O's rows with it
          ok = __all_sync(0xffffffffu, mbar_wait_bounded(&pv_done[(T - 1) & 3], ((T - 1) >> 2) & 1)) != 0;
          if (!ok) break;
          tc::fence_after();
          const float f = moves ? fast_exp2(m_ref - m_new) : 1.f;
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            uint32_t o[32];
            tc::ld32(tO + c0 + lane_off, o);
            tc::wait_ld();
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            tc::st32(tO + c0 + lane_off, o);
          }
          tc::wait_st();
        }
        s_m[(T & 3) * 128 + r] = m_new;
        __syncwarp();
        if (lane == 0) mbar_arrive(&m_bar[(T & 3) * 4 + quarter]);
        m_own = m_new;
        const float mm = m_new == -INFINITY ? 0.f : m_new, ms = m_sum == -INFINITY ? 0.f : m_sum;
        // Beside far larger values a tile's weights may be stored as nothing: their part of the sum is worked
        // out by itself.  (Without this branch the code about it came out slower: a whole prompt of 4,095 621 us.)
        const bool apart = __any_sync(0xffffffffu, mm - ms - e > LP_FAR && top != -INFINITY);
        if (apart) {
#pragma unroll 1
          for (int c0 = 0; c0 < LP_T; c0 += 32) {
            tc::ld32(tb + c0, s[0]);
            tc::wait_ld();
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < 32; ++c) sum += fast_exp2(fmaf(__uint_as_float(s[0][c]), sc, -ms));
            l += sum;
          }
        }
        const float shift = e - mm;
        const uint64_t cc = f32x2(shift, shift);
        uint64_t sum = f32x2(0.f, 0.f);
#pragma unroll 1
        for (int c0 = 0; c0 < LP_T; c0 += 64) {
          tc::ld32(tb + c0, s[0]);
          tc::ld32(tb + c0 + 32, s[1]);
          tc::wait_ld();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t p[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              float d0, d1;
              unpack_f32x2(fma_f32x2(f32x2(__uint_as_float(s[h][2 * c]), __uint_as_float(s[h][2 * c + 1])),
                                     kk, cc), d0, d1);
              const float p0 = fast_exp2(d0), p1 = fast_exp2(d1);
              p[c] = pack_f16x2(p0, p1);
              sum = add_f32x2(sum, f32x2(p0, p1));
            }
            st16(tb + c0 / 2 + 16 * h, p);   // over scores already read
          }
        }
        float u, v;
        unpack_f32x2(sum, u, v);
        if (i + 2 < nt) e_next = powers[i + 2];
        if (!apart) l = fmaf(u + v, fast_exp2(fminf(-ms - shift, 126.f)), l);
        tc::wait_st();
        tc::fence_before();
        __syncwarp();
        if (lane == 0) tc::arrive_cluster(&p_ready[T & 3], 0);
      }
      t0 += nt;
      const int last = t0 - 1;
      // The group with the last tile, whose reference is the row's, goes on to O; the other leaves it its
      // sum.  (Barriers and places of four segments in turn: neither group gets that far ahead.)
      float2* const ml = s_ml + (seg & 3) * 128 + r;
      if (group != (last & 1)) {
        *ml = make_float2(m_sum, l);
        asm volatile("bar.arrive %0, 256;\n" ::"r"(1 + (seg & 3)) : "memory");
        continue;
      }
      asm volatile("bar.sync %0, 256;\n" ::"r"(1 + (seg & 3)) : "memory");
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&pv_done[last & 3], (last >> 2) & 1)) != 0;
      if (!ok) continue;
      tc::fence_after();
      const float2 other = *ml;
      // no reference: a sum of zero, or NaN where every score was
      const float ms = fmaxf(m_sum, other.x);
      const float lsum = ms == -INFINITY ? l + other.y : l * fast_exp2(m_sum - ms) + other.y * fast_exp2(other.x - ms);
      const bool whole = nt == sg.n;
      const int64_t prow = ((int64_t)(2 * pair + (sg.j0 == 0 ? 1 : 0)) * LP_Q) + 128 * rank;
      float inv = whole ? (lsum != 0.f ? 1.f / lsum : 0.f) : 1.f, rest;
      const float half = half_power(m_own, ms, &rest);
      // a value that is not finite among those seen
      if (__reduce_min_sync(0xffffffffu, first_bad) <= limit) inv = __uint_as_float(0x7FC00000u);
      if (!whole) a.ml[prow + r] = make_float4(m_own, ms, lsum * inv, 0.f);
      inv *= half;
      // 128-byte pieces of a warp's 32 rows go through shared memory, so that whole lines are written
      const uint32_t tr = smem_u32(sm + L::OFF_OUT) + (warp - 4) * 4096;
      uint8_t* const to = whole ? reinterpret_cast<uint8_t*>(a.out + ((int64_t)row0 * a.H + a.h0 + sg.hl) * 128)
                                : reinterpret_cast<uint8_t*>(a.o + (prow + quarter * 32) * 128);
      const int64_t pitch = whole ? (int64_t)a.H * 256 : 512;
      uint32_t o[2][32], w[1][32];
      auto read = [&](int half) {   // 64 columns
        tc::ld32(tO + 64 * half + lane_off, o[0]);
        tc::ld32(tO + 64 * half + 32 + lane_off, o[1]);
        tc::wait_ld();
        if (half == 1) {   // the next segment's products may begin
          tc::fence_before();
          __syncwarp();
          if (lane == 0) tc::arrive_cluster(o_free, 0);
        }
      };
      auto out = [&](const uint32_t (&x)[32], int part) {   // 32 words a row
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sts128(tr + lane * 128 + ((k ^ (lane & 7)) << 4), x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int row = u * 4 + (lane >> 3), piece = lane & 7;
          const uint4 v = lds128(tr + row * 128 + ((piece ^ (row & 7)) << 4));
          if (row0 + row < a.C) *reinterpret_cast<uint4*>(to + row * pitch + part * 128 + piece * 16) = v;
        }
        __syncwarp();
      };
      if (whole) {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          read(half);
#pragma unroll
          for (int c = 0; c < 32; ++c)
            w[0][c] = pack_bf16x2(__uint_as_float(o[c >> 4][(2 * c) & 31]) * inv * rest,
                                  __uint_as_float(o[c >> 4][(2 * c + 1) & 31]) * inv * rest);
          out(w[0], half);
        }
      } else {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          read(half);
          out(o[0], 2 * half);
          out(o[1], 2 * half + 1);
        }
      }
    }
    if (!ok && lane == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
  }
  // Neither CTA may release TMEM or exit while its partner can still reach it.  CTA 1's arrivals were all waited
  // for, the last ones at the issuer's end, the products' at k_free, pv_done and q_free by the copies' last turns,
  // at s_full by the softmax.
  tc::fence_before();
  settle(ok);
  cluster_meet();
  if (warp == 0) {
    tc::fence_after();
    tc::dealloc2(*tmem_slot, 512);
  }
}

// ---------------------------------------------------------------------------
// Join the parts of the item that ends in pair p, if it began in one before: four rows a
// warp, a lane 4 channels.  Bound: the parts' way from L2 (18 MB for 128 items of 256 queries: 8.8 us).
// ---------------------------------------------------------------------------
constexpr int LJ_WARPS = 8, LJ_ROWS = 4, LJ_MAX = 128;   // LJ_MAX: pairs at most

__global__ void __launch_bounds__(32 * LJ_WARPS)
latent_prefill_merge_kernel(const __grid_constant__ LatentChunk a) {
  __shared__ float s_w[LJ_WARPS][LJ_ROWS][LJ_MAX];
  __shared__ int s_slot[LJ_MAX], s_n;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const int pair = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ChunkIter run = chunk_run(a, pair);
  const int64_t item = run.start;
  ChunkSeg sg;
  const bool joins = run.u0 < run.u1 && next_chunk_seg(a, run, sg) && sg.j0 > 0 && sg.j1 == sg.n;
  const int row0 = ((int)blockIdx.y * LJ_WARPS + warp) * LJ_ROWS;
  if (joins && warp == 0) {   // pairs from the first to this one that have units at all
    const PairRuns runs(a.units, a.pairs, a.inv);
    const int p0 = runs.of(item + LP_HDR);
    int n = 0;
    for (int p = p0 + lane; p - lane <= pair; p += 32) {
      const bool has = p <= pair && runs.first(p) < runs.first(p + 1);
      const unsigned m = __ballot_sync(0xffffffffu, has);
      if (has) s_slot[n + __popc(m & ((1u << lane) - 1))] = 2 * p + (p == p0 ? 1 : 0);
      n += __popc(m);
    }
    if (lane == 0) s_n = n;
  }
  // Blocks with nothing to join wait too: the kernel after this one takes this one's end for the end of
  // all before it.
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (!joins) return;
  __syncthreads();
  const int n = s_n, q0 = sg.qt * LP_Q + row0;
  if (q0 >= a.C) return;
  // the first parts, under way while the weights are worked out
  const float* const o = a.o + (int64_t)row0 * 128 + lane * 4;
  float4 v[2][LJ_ROWS];
  auto load = [&](int i) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int k = 0; k < LJ_ROWS; ++k)   // rows past the chunk's end: whatever is there
        if (i + u < n)
          v[u][k] = *reinterpret_cast<const float4*>(o + ((int64_t)s_slot[i + u] * LP_Q + k) * 128);
  };
  load(0);
  // weights: eight lanes a row
  const int sub = lane & 7, mine = lane >> 3;
  const float4* const ml = a.ml + row0 + mine;
  float M = -INFINITY, MS = -INFINITY, S = 0.f;
  for (int i = sub; i < n; i += 8) {
    const float4 x = ml[(int64_t)s_slot[i] * LP_Q];
    M = fmaxf(M, x.x);
    MS = fmaxf(MS, x.y);
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    MS = fmaxf(MS, __shfl_xor_sync(0xffffffffu, MS, o));
  }
  for (int i = sub; i < n; i += 8) {
    const float4 x = ml[(int64_t)s_slot[i] * LP_Q];
    s_w[warp][mine][i] = M == -INFINITY ? 1.f : fast_exp2(x.x - M);
    S = fmaf(MS == -INFINITY ? 1.f : fast_exp2(x.y - MS), x.z, S);
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
  __syncwarp();
  float4 acc[LJ_ROWS];
#pragma unroll
  for (int k = 0; k < LJ_ROWS; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < n; i += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int k = 0; k < LJ_ROWS; ++k)
        if (i + u < n) {
          const float w = s_w[warp][k][i + u];
          acc[k].x = fmaf(v[u][k].x, w, acc[k].x);
          acc[k].y = fmaf(v[u][k].y, w, acc[k].y);
          acc[k].z = fmaf(v[u][k].z, w, acc[k].z);
          acc[k].w = fmaf(v[u][k].w, w, acc[k].w);
        }
    load(i + 2);
  }
#pragma unroll
  for (int k = 0; k < LJ_ROWS; ++k) {
    const float s = __shfl_sync(0xffffffffu, S, 8 * k);
    float rest;
    const float half = half_power(__shfl_sync(0xffffffffu, M, 8 * k), __shfl_sync(0xffffffffu, MS, 8 * k), &rest);
    const float inv = (s != 0.f ? 1.f / s : 0.f) * half;
    if (q0 + k < a.C)
      *reinterpret_cast<uint2*>(a.out + ((int64_t)(q0 + k) * a.H + a.h0 + sg.hl) * 128 + lane * 4) =
          make_uint2(pack_bf16x2(acc[k].x * inv * rest, acc[k].y * inv * rest),
                     pack_bf16x2(acc[k].z * inv * rest, acc[k].w * inv * rest));
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
int latent_query_map(const void* q, int64_t H, int64_t C, CUtensorMap* map);

// Heads a pass: enough for eight items a pair, and at least what the L2 cache holds of their keys
// and values, but no more than 1 GB of them (one head, whatever it takes).
static int64_t heads_per_pass(int64_t n_pad, int64_t C, int64_t H, int64_t pairs) {
  const int64_t bytes = n_pad * 512, q_tiles = (C + LP_Q - 1) / LP_Q;
  const int64_t cached = (int64_t)96 * 1024 * 1024 / bytes, most = (int64_t)1024 * 1024 * 1024 / bytes;
  int64_t h = (8 * pairs + q_tiles - 1) / q_tiles;
  if (h > most) h = most;
  if (h < cached) h = cached;
  if (h < 1) h = 1;
  if (h >= H) return H;
  const int64_t passes = (H + h - 1) / h;   // passes of about equal size
  return (H + passes - 1) / passes;
}

static int64_t padded(int64_t n) { return (n + 255) / 256 * 256; }

// what a pass of so many heads takes
static size_t pass_bytes(int64_t n_pad, int64_t heads, int64_t pairs) {
  return (size_t)(256 + round256(heads * n_pad / 8) + round256(heads * n_pad / 32) + 2 * pairs * LP_Q * (16 + 512) +
                  heads * n_pad * 512);
}

size_t latent_prefill_workspace_bytes(int64_t q_start, int64_t C, int64_t H, int64_t sms) {
  const int64_t pairs = sms / 2, n_pad = padded(q_start + C);
  return C == 0 ? 256 : pass_bytes(n_pad, heads_per_pass(n_pad, C, H, pairs), pairs);
}

template <typename... P, typename... A>
static int launch(void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t stream, const A&... args) {
  if (smem && smem_optin((const void*)kernel, smem) != JF_OK) return JF_ERR_CUDA;
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

int launch_latent_prefill(const LatentPrefill& p, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  const int pairs = sm_count() / 2;
  if (pairs > LJ_MAX) return JF_ERR_UNSUPPORTED;
  LatentChunk a{};
  a.pool = p.pool;
  a.pt = p.pt;
  a.out = p.out;
  a.status = p.status;
  a.n = p.q_start + p.C;
  const int64_t n_pad = padded(a.n);
  a.n_pad = (int32_t)n_pad;
  a.q_start = p.q_start;
  a.C = p.C;
  a.H = p.H;
  a.causal = p.causal != 0;
  a.pairs = pairs;
  a.inv = pairs_inverse(pairs);
  a.scale_log2 = p.scale_log2;
  const int64_t q_tiles = ((int64_t)p.C + LP_Q - 1) / LP_Q;
  a.q_tiles = (int32_t)q_tiles;
  const int64_t tiles = ((int64_t)a.n + LP_T - 1) / LP_T, before = ((int64_t)p.q_start + LP_T - 1) / LP_T;
  // as chunk_start() has it, and the last query tile's
  a.units_head = (a.causal ? (q_tiles - 1) * (q_tiles - 2) + (q_tiles - 1) * (2 + before + LP_HDR)
                           : (q_tiles - 1) * (tiles + LP_HDR)) + tiles + LP_HDR;
  // The caller's workspace may be one for another chunk of the same prompt, and that a smaller one: a short chunk
  // takes more heads at a time than a long one.
  int64_t per = heads_per_pass(n_pad, p.C, p.H, pairs);
  while (per > 1 && pass_bytes(n_pad, per, pairs) > workspace_bytes) --per;
  uint8_t* ws = static_cast<uint8_t*>(workspace) + 256;
  a.bad = reinterpret_cast<int32_t*>(ws);
  ws += round256(per * n_pad / 8);
  a.power = reinterpret_cast<float*>(ws);
  ws += round256(per * n_pad / 32);
  a.ml = reinterpret_cast<float4*>(ws);
  ws += (int64_t)2 * pairs * LP_Q * 16;
  a.o = reinterpret_cast<float*>(ws);
  ws += (int64_t)2 * pairs * LP_Q * 512;
  a.k = reinterpret_cast<uint16_t*>(ws);
  a.v = a.k + per * n_pad * 128;
  CUtensorMap pmap, wkmap, wvmap, qmap, kmap, vmap;
  int st = bf16_rows_map(p.pool.base, p.pool.row, p.pool.num_pages * p.pool.P, 64, &pmap);
  if (!st) st = bf16_rows_map(p.w_k, p.pool.R, (int64_t)p.H * 128, 128, &wkmap);
  if (!st) st = bf16_rows_map(p.w_v, p.pool.R, (int64_t)p.H * 128, 128, &wvmap);
  if (!st) st = latent_query_map(p.q, p.H, p.C, &qmap);
  if (!st) st = bf16_rows_map(a.k, 128, per * n_pad, 64, &kmap);
  if (!st) st = bf16_rows_map(a.v, 128, per * n_pad, 128, &vmap);
  if (st) return st;
  for (int64_t h0 = 0; h0 < p.H; h0 += per) {
    a.h0 = (int32_t)h0;
    a.heads = (int32_t)(p.H - h0 < per ? p.H - h0 : per);
    a.units = a.units_head * a.heads;
    const int64_t e_tiles = n_pad / 256 * a.heads;
    const unsigned e_pairs = (unsigned)(e_tiles < pairs ? e_tiles : pairs);
    st = launch(latent_expand_kernel, dim3(2 * e_pairs), LE_THREADS, LeSmem::TOTAL, stream, pmap, wkmap,
                wvmap, a);
    if (!st)
      st = launch(latent_prefill_kernel, dim3(2 * (unsigned)pairs), LA_THREADS, LaSmem::TOTAL, stream, qmap,
                  pmap, kmap, vmap, a);
    if (!st)
      st = launch(latent_prefill_merge_kernel, dim3((unsigned)pairs, LP_Q / (LJ_WARPS * LJ_ROWS)), 32 * LJ_WARPS, 0,
                  stream, a);
    if (st) return st;
  }
  return JF_OK;
}

}  // namespace jfkv
