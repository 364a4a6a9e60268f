// Decode attention over the latent cache on the 5th-generation tensor cores: one
// query a request, or groups of requests over a shared prefix.
//
// All heads read the same position rows, so up to 128 (request, head) rows form one
// M = 128 tile of a CTA pair: S = Q K^T with K = (c, r) of R + 64 channels, O += P V
// with V = c.  Each CTA of the pair holds 64 query rows and gets their S and O; of
// the products' other operand it supplies half: of a tile of 128 positions its own
// 64 rows of K, and its own R / 2 channels of V.  In tensor memory an M = 128 pair
// product keeps columns 0 .. N/2 - 1 in lanes 0 - 63 and the others in lanes 64 - 127,
// so O takes R / 2 columns, and a row is four threads' of the eight softmax warps.
//
// Work: the calls' items (a group's rows over its prefix, a request's heads over its
// own positions), in tiles and a header each, are laid end to end and cut into one
// run of equal length per CTA pair, whatever the lengths.  An item that one pair
// takes whole is written out directly (decode) or as one partial (prefixes); of one
// that is cut each pair writes an unnormalized partial (m, l, O), and a second kernel
// joins them.  A pair has at most two cut items, so the workspace does not depend on
// any length.
//
// What bounds it: memory, the products and what of one the other cannot hide.  32 requests to
// 65,535 positions x 16 heads take 99 to 104 us: their 593 MB 87 at copy rate, the same launch without
// its loads 80 (2,500 cycles a tile of R = 512 where its products are 2,176).  All of K's and V's
// shared memory holds one tile each, the next one's K is on its way into the L2 cache, and every
// position crosses from there twice, as K and as V: 137 KB a tile and CTA, 12 TB/s in all.  One
// request of 131,072 positions x 128 heads takes 41 us: a tile passes at memory's rate (1.68 us;
// 22.2 for all), before it the plan and the first copies, after it 128 rows x R of every pair
// go out (2.6) and are joined (6).  Short calls are latency: 10.0 us for one request of 4,096 positions
// are the plan (1.0 us), a page's look-up, the copies and S (1.9), softmax and P V (1.3), O out
// (1.0), and set-up, two launches and the join (4.8).
//
// Warp roles (each CTA):
//   warp 0     TMEM; CTA 0: issues the pair's MMAs; CTA 1: passes its K and Q arrivals on
//   warp 1     K by TMA
//   warp 2     passes V's arrivals on; where a tile's last positions hold nothing yet it
//              first clears them (a weight of zero does not undo a NaN)
//   warp 3     V by TMA
//   warps 4-11 softmax (four threads a row), O out; a segment's last P V done, 128 rows x R / 2
//              columns leave in 2.6 us, 16 rows in 0.9
//   warp 12    Q by TMA, as soon as the last products with the segment's before are done
#include <cmath>

#include "latent_tc.cuh"

namespace jfkv {

constexpr int LD_T = 128;           // positions a tile
constexpr int LD_ROWS = 128;        // rows a pair, 64 each CTA
// An item's fixed cost in tiles, its queries' way in and its partials' way out: more where both CTAs have
// rows.  (2 x 4 continuations x 128 heads 21.8 us with 4 there, 23.9 with 2; 64 continuations x 16 heads
// 56.4 and 57.0.)
constexpr int LD_HDR = 2, LD_HDR_FULL = 4;
constexpr int LD_THREADS = 32 * 13;
constexpr int LD_SOFT = 8;           // softmax warps
constexpr int LD_SBUF = 4;          // S buffers: S may be this many tiles ahead of P V
constexpr float LD_TOP = 16.f;      // the reference maximum moves when a score exceeds it by this (log2)

struct LatentPlan {
  int32_t pairs;                    // CTA pairs of the launch
  int32_t items, prefix_items, blocks;   // items; those of prefixes; row blocks of a request
  int32_t slot_rows;                // rows of a cut item's partial
  uint32_t inv;                     // of the pairs, for PairRuns
  int32_t item0[LAT_MAX_GROUPS + 1];     // first items of the groups
  int64_t* units;                   // of the call, for the joins
  int2* spans;                      // [items] first and last pair of its tiles, (0, -1) where it has none
  float* ml;                        // [rows][2]
  float* o;                         // [rows][R]
};

template <int R>
struct LdSmem {
  static constexpr int KC = R == 512 ? 3 : 5;          // 64-channel chunks of K a stage
  static constexpr int KPT = (R / 64 + 1) / KC;        // stages a tile
  static constexpr int KS = R == 512 ? 3 : 2;          // K stages
  static constexpr int U = R / 256;                    // V stages a tile (256 channels of the pair)
  static constexpr int VS = 2;                         // V stages
  static constexpr int CHUNK = 64 * 128;               // 64 rows of 128 bytes
  static constexpr int Q_BYTES = (R / 64 + 1) * CHUNK;
  static constexpr int K_BYTES = KC * CHUNK;
  static constexpr int V_BYTES = 2 * 2 * CHUNK;        // [2 x 64 positions][2 x 64 channels][64][128 B]
  static constexpr int OFF_K = Q_BYTES;
  static constexpr int OFF_V = OFF_K + KS * K_BYTES;
  static constexpr int OFF_P = OFF_V + VS * V_BYTES;   // [2 x 64 positions][64 rows][128 B]
  static constexpr int OFF_BAR = OFF_P + 2 * CHUNK;
  static constexpr int OFF_X = OFF_BAR + 256;          // [2][256] exchange between a row's threads
  static constexpr int OFF_PLAN = OFF_X + 2 * 256 * 4; // [16] of the plan's scan
  static constexpr int OFF_FIRST = OFF_PLAN + 16 * 8;  // LdFirst
  static constexpr int TOTAL = OFF_FIRST + 16;
  static_assert(TOTAL <= 227 * 1024, "shared memory per CTA");
};

// ---- items ------------------------------------------------------------------------
struct LatentItem {
  const int32_t* pt;
  int32_t len, row0, nrows;
};

__device__ __forceinline__ int request_of(const LatentPlan& pl, int k) {
  return pl.blocks == 1 ? k : k / pl.blocks;
}
// the group of item i, -1 for a request's own positions
__device__ __forceinline__ int item_group(const LatentPlan& pl, int i) {
  if (i >= pl.prefix_items) return -1;
  int g = 0;
  while (pl.item0[g + 1] <= i) ++g;
  return g;
}
// its positions, -1 where their number does not fit the table
__device__ __forceinline__ int item_len(const LatentDecode& a, const LatentPlan& pl, int i, int g) {
  const int n = g >= 0 ? a.prefix_lens[g] : a.context_lens[request_of(pl, i - pl.prefix_items)];
  const int stride = g >= 0 ? a.prefix_stride : a.pt_stride;
  return n < 0 || n > (int64_t)stride * a.pool.P || n > JF_LATENT_MAX_POSITIONS ? -1 : n;
}

__device__ __forceinline__ int item_alone(const LatentPlan& pl, int g) {
  return g >= 0 ? pl.item0[g + 1] - pl.item0[g] == 1 : pl.blocks == 1;
}

__device__ __forceinline__ int tiles_of(int len) { return len <= 0 ? 0 : (len + LD_T - 1) / LD_T; }
__device__ __forceinline__ int header_of(const LatentDecode& a, int g) {
  return g >= 0 || a.H > LD_ROWS / 2 ? LD_HDR_FULL : LD_HDR;
}
__device__ __forceinline__ int64_t units_of(const LatentDecode& a, int g, int len) {
  const int n = tiles_of(len);
  return n ? n + header_of(a, g) : 0;
}

__device__ __forceinline__ LatentItem item_of(const LatentDecode& a, const LatentPlan& pl, int i,
                                              int g, int len) {
  LatentItem it;
  it.len = len;
  if (g >= 0) {
    it.row0 = a.first[g] * a.H + (i - pl.item0[g]) * LD_ROWS;
    it.nrows = min(LD_ROWS, a.first[g + 1] * a.H - it.row0);
    it.pt = a.prefix_table + (int64_t)g * a.prefix_stride;
  } else {
    const int k = i - pl.prefix_items, b = request_of(pl, k), hb = k - b * pl.blocks;
    it.row0 = b * a.H + hb * LD_ROWS;
    it.nrows = min(LD_ROWS, a.H - hb * LD_ROWS);
    it.pt = a.page_table + (int64_t)b * a.pt_stride;
  }
  return it;
}

// The segments of a pair's run of units [u0, u1), in order.
struct Seg {
  LatentItem it;
  int item, j0, j1, n;   // tiles j0 .. j1 - 1 of the item's n
  int alone;             // no other item reads these positions
};
struct SegIter {
  int64_t start, u0, u1;   // first unit of the item
  int item;
  int len;                 // of the item, where it is known already (else LD_ASK)
};
constexpr int LD_ASK = -2;

__device__ __forceinline__ bool next_seg(const LatentDecode& a, const LatentPlan& pl, SegIter& s,
                                         Seg& seg) {
  while (s.item < pl.items && s.start < s.u1) {
    const int g = item_group(pl, s.item);
    const int len = s.len != LD_ASK ? s.len : item_len(a, pl, s.item, g);
    s.len = LD_ASK;
    const int n = tiles_of(len);
    const int64_t first = s.start + header_of(a, g);   // unit of tile 0
    const int64_t lo = max((int64_t)0, s.u0 - first), hi = min((int64_t)n, s.u1 - first);
    const int i = s.item++;
    if (n) s.start += n + header_of(a, g);
    if (lo < hi) {
      seg.it = item_of(a, pl, i, g, len);
      seg.item = i;
      seg.j0 = (int)lo;
      seg.j1 = (int)hi;
      seg.n = n;
      seg.alone = item_alone(pl, g);
      return true;
    }
  }
  return false;
}

// The segments after the first, by a call: one copy of the code for all roles, which then fit the
// instruction caches better (64 continuations x 16 heads 57.7 us with a copy each, 55.6 so; 4,096 requests of
// 64 positions x 16 heads 350 and 290).
struct SegStep {
  SegIter it;
  Seg seg;
  bool more;
};
__device__ __noinline__ SegStep far_seg(const LatentDecode& a, const LatentPlan& pl, SegIter s) {
  SegStep r;
  r.more = next_seg(a, pl, s, r.seg);
  r.it = s;
  return r;
}
__device__ __forceinline__ bool later_seg(const LatentDecode& a, const LatentPlan& pl, SegIter& s, Seg& seg) {
  if (s.item >= pl.items || s.start >= s.u1) return false;
  const SegStep r = far_seg(a, pl, s);
  s = r.it;
  seg = r.seg;
  return r.more;
}

struct LdFirst {   // a pair's first item
  int64_t start;
  int item, len;
};

// This pair's run of the items, which the last thread with items' units before it works out; every
// thread takes part.  Block 0 writes down the items' pairs for the kernel that joins the partials.
__device__ __forceinline__ SegIter plan_run(const LatentDecode& a, const LatentPlan& pl, int pair, int warp,
                                            int lane, int64_t* s_plan, LdFirst* s_first) {
  SegIter run{0, 0, 0, pl.items, LD_ASK};
  if (pl.items <= 32) {   // an item a lane, each warp by itself
    const int g = item_group(pl, lane);
    const int len = lane < pl.items ? item_len(a, pl, lane, g) : 0;
    const int n = (int)units_of(a, g, len);
    int incl = n;   // below 2^30
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const int at = incl - n;
    const PairRuns runs(__shfl_sync(0xffffffffu, incl, 31), pl.pairs, pl.inv);
    const int64_t u0 = runs.first(pair), u1 = runs.first(pair + 1);
    const unsigned mine = __ballot_sync(0xffffffffu, u0 < u1 && at <= u0 && u0 < incl);
    const int src = mine ? __ffs(mine) - 1 : 0;
    const int start = __shfl_sync(0xffffffffu, at, src), first_len = __shfl_sync(0xffffffffu, len, src);
    if (mine) run = SegIter{start, u0, u1, src, first_len};
    if (blockIdx.x == 0 && warp == 2) {   // which is the last to have anything else to do
      if (len < 0) flag_error(a.status, JF_DEV_ERR_POSITION);
      if (lane < pl.items) {
        int2 span = make_int2(0, -1);
        if (n) span = make_int2(runs.of(at + header_of(a, g)), runs.of(incl - 1));
        pl.spans[lane] = span;
      }
      if (lane == 31) *pl.units = incl;
    }
    return run;
  }
  const int per = (pl.items + LD_THREADS - 1) / LD_THREADS;
  const int i0 = min(pl.items, (int)threadIdx.x * per), i1 = min(pl.items, i0 + per);
  int64_t sum = 0;
  for (int i = i0; i < i1; ++i) {
    const int g = item_group(pl, i), len = item_len(a, pl, i, g);
    if (len < 0 && blockIdx.x == 0) flag_error(a.status, JF_DEV_ERR_POSITION);
    sum += units_of(a, g, len);
  }
  int64_t incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) s_plan[warp] = incl;
  if (threadIdx.x == 0) s_first->item = -1;
  __syncthreads();
  int64_t before = 0, units = 0;
#pragma unroll 1
  for (int w = 0; w < LD_THREADS / 32; ++w) {
    if (w < warp) before += s_plan[w];
    units += s_plan[w];
  }
  int64_t at = before + incl - sum;   // units before this thread's items
  const PairRuns runs(units, pl.pairs, pl.inv);
  const int64_t u0 = runs.first(pair), u1 = runs.first(pair + 1);
  const bool mine = u0 < u1 && at <= u0 && u0 < at + sum;
  int p = blockIdx.x == 0 && sum ? runs.of(at) : 0;   // the pair that has the unit looked at
  auto pair_of = [&](int64_t u) {
    while (runs.first(p + 1) <= u) ++p;
    return p;
  };
  if (mine || blockIdx.x == 0)
    for (int i = i0; i < i1; ++i) {
      const int g = item_group(pl, i), len = item_len(a, pl, i, g);
      const int64_t next = at + units_of(a, g, len);
      if (blockIdx.x == 0) {
        int2 span = make_int2(0, -1);
        if (next > at) {
          span.x = pair_of(at + header_of(a, g));
          span.y = pair_of(next - 1);
        }
        pl.spans[i] = span;
      }
      if (mine && at <= u0 && u0 < next) *s_first = LdFirst{at, i, len};
      at = next;
    }
  if (blockIdx.x == 0 && threadIdx.x == 0) *pl.units = units;
  __syncthreads();
  if (s_first->item >= 0) run = SegIter{s_first->start, u0, u1, s_first->item, s_first->len};
  return run;
}

template <int R>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LD_THREADS, 1)
latent_decode_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                     const __grid_constant__ CUtensorMap qmap, const __grid_constant__ LatentDecode a,
                     const __grid_constant__ LatentPlan pl) {
  using L = LdSmem<R>;
  constexpr uint32_t IDQK = idesc_bf16(LD_ROWS, LD_T, 0);
  constexpr uint32_t IDPV = idesc_bf16(LD_ROWS, 256, 1);
  extern __shared__ __align__(1024) uint8_t sm[];
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sm + L::OFF_BAR);
  // on CTA 0, where the pair's MMAs are issued:
  uint64_t* const k_full = bars + 0;     // [3] both CTAs' K of a stage
  uint64_t* const v_full = bars + 3;     // [2] both CTAs' V of a stage
  uint64_t* const p_ready = bars + 5;    // both CTAs' P of a tile
  uint64_t* const q_full = bars + 6;     // both CTAs' Q of a segment
  // on each CTA:
  uint64_t* const k_land = bars + 7;     // [3] CTA 1: its K
  uint64_t* const v_land = bars + 10;    // [2] its V
  uint64_t* const k_free = bars + 12;    // [3] stage read by its products
  uint64_t* const v_free = bars + 15;    // [2]
  uint64_t* const s_full = bars + 17;    // [4] S of tile t % 4
  uint64_t* const pv_done = bars + 21;   // P V of a tile
  uint64_t* const q_land = bars + 22;    // CTA 1: its Q
  uint64_t* const q_free = bars + 23;    // products with a segment's Q done
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 24);
  float* const s_x = reinterpret_cast<float*>(sm + L::OFF_X);
  int64_t* const s_plan = reinterpret_cast<int64_t*>(sm + L::OFF_PLAN);
  LdFirst* const s_first = reinterpret_cast<LdFirst*>(sm + L::OFF_FIRST);
  static_assert(sizeof(LdFirst) <= 16 && LD_THREADS / 32 <= 16, "shared memory of the plan");

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);   // uniform
  const int lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  const int pair = (int)(blockIdx.x >> 1);
  if (threadIdx.x == 0) {
    prefetch_tensormap(&kmap);
    prefetch_tensormap(&vmap);
    prefetch_tensormap(&qmap);
    for (int i = 0; i < 3; ++i) {
      mbar_init(&k_full[i], 2);
      mbar_init(&k_land[i], 1);
      mbar_init(&k_free[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&v_full[i], 2);
      mbar_init(&v_land[i], 1);
      mbar_init(&v_free[i], 1);
    }
    for (int i = 0; i < LD_SBUF; ++i) mbar_init(&s_full[i], 1);
    mbar_init(p_ready, 2 * LD_SOFT);
    mbar_init(q_full, 2);
    mbar_init(q_land, 1);
    mbar_init(q_free, 1);
    mbar_init(pv_done, 1);
    fence_barrier_init();
  }
  if (warp == 0) tc::alloc2(tmem_slot, 512);
  tc::fence_before();
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");   // waited for after the plan
  asm volatile("griddepcontrol.wait;\n" ::: "memory");   // what came before has been written

  // The first segment is worked out here, in one copy of that code for all roles: it is fetched when it
  // first runs (the roles' own copies took 2,000 to 2,500 cycles for it, 1 us).
  SegIter run = plan_run(a, pl, pair, warp, lane, s_plan, s_first);
  if (smem_u32(sm) & 1023u) {   // the swizzled layouts need it: no work, but the plan stands, which the joins read
    if (threadIdx.x == 0) flag_error(a.status, JF_DEV_ERR_LAYOUT);
    run.item = pl.items;
  }
  Seg sg;
  bool more = next_seg(a, pl, run, sg);
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");   // both CTAs: barriers, TMEM
  tc::fence_after();
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  // all 512 columns are this CTA's: O from 0, the S buffers behind it
  constexpr uint32_t tO = 0, tS = R / 2;

  bool ok = true;
  if (warp == 0) {
    if (rank == 0) {
      // ================= MMA issuer =================
      const uint32_t leader = elect_one();
      const uint64_t qd = tc::sdesc_sw128(smem_u32(sm), 16, 1024);
      const uint64_t kd = tc::sdesc_sw128(smem_u32(sm + L::OFF_K), 16, 1024);
      const uint64_t vd = tc::sdesc_sw128(smem_u32(sm + L::OFF_V), L::CHUNK, 1024);
      const uint64_t pd = tc::sdesc_sw128(smem_u32(sm + L::OFF_P), 16, 1024);
      auto wait = [&](uint64_t* bar, int phase) {
        return __all_sync(0xffffffffu, mbar_wait_bounded(bar, phase & 1)) != 0;
      };
      // Whichever product has its operands goes next: taken in a fixed order, S behind K that is on its
      // way from memory held up P V whose V stage is wanted for the next tile.  S buffers bound how
      // far S may be ahead.
      int ks = 0, kp = 0, vs = 0, vp = 0;   // next stage of K and of V, and how often their rings went round
      int t = 0, nseg = 0;                 // tiles and segments of all segments so far
      // tiles of the next segment, or the next two: arrivals are asked for where a copy will wait for them, so
      // that none is on its way when the pair parts (copies that waited for the last ones at their ends
      // instead took one request of 4,096 positions from 10.1 to 10.8 us: more code to fetch)
      constexpr int D = L::KS / L::KPT;    // tiles that the rings hold
      static_assert(D == L::VS / L::U && D <= 2, "one look ahead for both rings");
      auto tiles = [&](bool is) { return __all_sync(0xffffffffu, is) ? __shfl_sync(0xffffffffu, sg.j1 - sg.j0, 0) : 0; };
      int next = tiles(more), next2 = 0;
      if (D == 2) next2 = tiles(later_seg(a, pl, run, sg));
      auto ready = [&](uint64_t* bar, int phase) {
        return __all_sync(0xffffffffu, mbar_test(bar, phase)) != 0;
      };
      while (ok && next > 0) {
        ok = wait(q_full, nseg);
        ++nseg;
        const int nt = next;
        if (D == 2) next = next2;
        (D == 2 ? next2 : next) = tiles(later_seg(a, pl, run, sg));
        const int again = nt - D + next + next2;   // tiles whose stages will be filled again
        int qi = 0, qc = 0, pi = 0, pu = 0;   // next S (tile, stage) and P V (tile, stage)
        uint32_t idle = 0;
        while (ok && pi < nt) {
          bool did = false;
          if (qi < nt && qi - pi < LD_SBUF && ready(&k_full[ks], kp)) {
            tc::fence_after();
            const uint64_t q0 = qd + (uint64_t)(qc * (L::K_BYTES >> 4));
            const uint64_t k0 = kd + (uint64_t)(ks * (L::K_BYTES >> 4));
            const uint32_t d = tS + ((t + qi) % LD_SBUF) * 64;
#pragma unroll
            for (int k = 0; k < 4 * L::KC; ++k) {
              const uint32_t at = ((k >> 2) * L::CHUNK + (k & 3) * 32) >> 4;
              mma2_ss_if(leader, d, q0 + at, k0 + at, IDQK, (qc > 0 || k > 0) ? 1u : 0u);
            }
            tc::commit2_both_if(qi < again ? leader : 0u, &k_free[ks]);
            if (++ks == L::KS) {
              ks = 0;
              ++kp;
            }
            if (++qc == L::KPT) {
              tc::commit2_both_if(leader, &s_full[(t + qi) % LD_SBUF]);
              if (qi == nt - 1) tc::commit2_both_if(next > 0 ? leader : 0u, q_free);
              qc = 0;
              ++qi;
            }
            did = true;
          }
          if (pi < qi && (pu > 0 || ready(p_ready, t + pi)) && ready(&v_full[vs], vp)) {
            tc::fence_after();
            const uint64_t v0 = vd + (uint64_t)(vs * (L::V_BYTES >> 4));
            const uint32_t d = tO + pu * 128;
#pragma unroll
            for (int k = 0; k < LD_T / 16; ++k)
              mma2_ss_if(leader, d, pd + (((k >> 2) * L::CHUNK + (k & 3) * 32) >> 4),
                         v0 + (((k >> 2) * 2 * L::CHUNK + (k & 3) * 2048) >> 4), IDPV, (pi > 0 || k > 0) ? 1u : 0u);
            tc::commit2_both_if(pi < again ? leader : 0u, &v_free[vs]);
            if (++vs == L::VS) {
              vs = 0;
              ++vp;
            }
            if (++pu == L::U) {
              tc::commit2_both_if(leader, pv_done);
              pu = 0;
              ++pi;
            }
            did = true;
          }
          idle = did ? 0 : idle + 1;
          if (idle > (1u << 24)) ok = false;
        }
        t += nt;
      }
        __syncwarp();
    } else {
      // ================= CTA 1's Q and K arrivals =================
      if (lane == 0) {
        int ks = 0, nseg = 0;
        for (; ok && more; more = later_seg(a, pl, run, sg)) {
          ok = mbar_wait_bounded(q_land, nseg & 1);
          if (ok) tc::arrive_cluster(q_full, 0);
          ++nseg;
          for (int i = (sg.j1 - sg.j0) * L::KPT; i > 0 && ok; --i, ++ks) {
            ok = mbar_wait_bounded(&k_land[ks % L::KS], (ks / L::KS) & 1);
            if (ok) tc::arrive_cluster(&k_full[ks % L::KS], 0);
          }
        }
        }
      __syncwarp();
    }
  } else if (warp == 1) {
    // ================= K: this CTA's 64 positions of each tile =================
    if (lane == 0) {
      int ks = 0;
      const int last = (int)(a.pool.num_pages << a.pool.log2P);   // no row
      for (; ok && more; more = later_seg(a, pl, run, sg)) {
        int y = half_row(a.pool, sg.it.pt, sg.j0 * LD_T + 64 * (int)rank, sg.it.len, a.status);
        for (int j = sg.j0; j < sg.j1 && ok; ++j) {
          const int row = y;
          if (j + 1 < sg.j1)
            y = half_row(a.pool, sg.it.pt, (j + 1) * LD_T + 64 * (int)rank, sg.it.len, a.status);
          const int apos = (j + 1) * LD_T + 64 * (int)rank, ahead_rows = sg.it.len - apos;
          const int ahead = j + 1 < sg.j1 && sg.alone ? y : last;
          for (int c = 0; c < L::KPT; ++c, ++ks) {
            const int st = ks % L::KS;
            if (ks >= L::KS && !mbar_wait_bounded(&k_free[st], (ks / L::KS - 1) & 1)) {
              ok = false;
              break;
            }
            uint64_t* const land = rank == 0 ? &k_full[st] : &k_land[st];
            mbar_arrive_expect_tx(land, L::K_BYTES);
            tma_load_3d(smem_u32(sm + L::OFF_K + st * L::K_BYTES), &kmap, 0, row, c * L::KC, land);
            // The ring holds one tile, less than memory's latency calls for: what comes after it is brought
            // into the L2 cache meanwhile (from where V is read as well), a part with every stage.
            if (ahead < last) {
              const int r0 = c * (64 / L::KPT), rows = min(c + 1 == L::KPT ? 64 - r0 : 64 / L::KPT, ahead_rows - r0);
              if (rows > 0)
                prefetch_l2(a.pool.base + (int64_t)(ahead + r0) * (R + LAT_ROT), (uint32_t)rows * (R + LAT_ROT) * 2);
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ================= V's arrivals; positions past the last one cleared =================
    int vs = 0;
    for (; ok && more; more = later_seg(a, pl, run, sg))
      for (int j = sg.j0; j < sg.j1 && ok; ++j) {
        const int live = sg.it.len - j * LD_T;   // positions of this tile that there are
        for (int u = 0; u < L::U; ++u, ++vs) {
          const int st = vs % L::VS;
          if (!mbar_wait_bounded(&v_land[st], (vs / L::VS) & 1)) {
            ok = false;
            break;
          }
          if (live < LD_T && (live & 63)) {   // past the half's end the copy brought zeros
            const uint32_t at = smem_u32(sm + L::OFF_V + st * L::V_BYTES + (live >> 6) * 2 * L::CHUNK);
            for (int p = (live & 63) * 8 + lane; p < 64 * 8; p += 32)
              for (int ch = 0; ch < 2; ++ch) sts128(at + ch * L::CHUNK + p * 16, 0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
          }
          __syncwarp();
          if (lane == 0) tc::arrive_cluster(&v_full[st], 0);
        }
      }
  } else if (warp == 3) {
    // ================= V: this CTA's channels of all 128 positions =================
    if (lane == 0) {
      int vs = 0;
      for (; ok && more; more = later_seg(a, pl, run, sg))
        for (int j = sg.j0; j < sg.j1 && ok; ++j) {
          int row[2];
          for (int h = 0; h < 2; ++h)
            row[h] = half_row(a.pool, sg.it.pt, j * LD_T + 64 * h, sg.it.len, nullptr);
          for (int u = 0; u < L::U; ++u, ++vs) {
            const int st = vs % L::VS;
            if (vs >= L::VS && !mbar_wait_bounded(&v_free[st], (vs / L::VS - 1) & 1)) {
              ok = false;
              break;
            }
            mbar_arrive_expect_tx(&v_land[st], L::V_BYTES);
            for (int h = 0; h < 2; ++h)
              tma_load_3d(smem_u32(sm + L::OFF_V + st * L::V_BYTES + h * 2 * L::CHUNK), &vmap, 0, row[h],
                          u * 4 + (int)rank * 2, &v_land[st]);
          }
        }
    }
    __syncwarp();
  } else if (warp == 4 + LD_SOFT) {
    // ================= Q: 64 rows from the item's first; rows past its last are computed and not
    // stored =================
    if (lane == 0) {
      // (a barrier of its own: one that other tiles complete as well could be a phase behind, and its
      // parity then says yes too early)
      int nseg = 0;
      for (; ok && more; more = later_seg(a, pl, run, sg)) {
        if (nseg > 0 && !mbar_wait_bounded(q_free, (nseg - 1) & 1)) {
          ok = false;
          break;
        }
        ++nseg;
        uint64_t* const land = rank == 0 ? q_full : q_land;
        mbar_arrive_expect_tx(land, L::Q_BYTES);
        for (int c = 0; c < L::KPT; ++c)
          tma_load_3d(smem_u32(sm) + c * L::K_BYTES, &qmap, 0, sg.it.row0 + 64 * (int)rank, c * L::KC, land);
      }
    }
    __syncwarp();
  } else {
    // ================= softmax, O =================
    // Four threads have a row: of its lane with the tile's first 64 positions and the one with the
    // others, each half of the 64 (and half of O's columns of that lane).
    const int quarter = warp & 3, half = quarter >> 1, side = warp >= 4 + LD_SOFT / 2 ? 1 : 0;
    const int r = (quarter & 1) * 32 + lane;
    const int tid = (int)threadIdx.x - 4 * 32;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t sp = smem_u32(sm + L::OFF_P);
    // the four warps that hold the same rows
    auto row_sync = [&] { asm volatile("bar.sync %0, 128;\n" ::"r"(1 + (quarter & 1)) : "memory"); };
    // weights are 2^(sc S - m), sc above zero: a scale below it negates S first, one of zero makes it
    // zero (or NaN)
    const float sc = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
    const int end = (int)(a.pool.num_pages << a.pool.log2P);
    // positions of this thread's 32 in tile j that there are
    auto live_of = [&](const Seg& g, int j) {
      const int pos = j * LD_T + half * 64;
      return half_row(a.pool, g.it.pt, pos, g.it.len, nullptr) == end ? 0 : g.it.len - pos - side * 32;
    };
    int t = 0;
    Seg nx;
    // A wait that gave up ends the work but not the meetings: the warps of a row would wait for one
    // another for ever.
    while (more) {
      float m = -INFINITY, l = 0.f;
      int live = live_of(sg, sg.j0);
      for (int j = sg.j0; j < sg.j1; ++j, ++t) {
        ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&s_full[t % LD_SBUF], (t / LD_SBUF) & 1)) != 0;
        tc::fence_after();
        uint32_t s[32];
        tc::ld32(tS + (t % LD_SBUF) * 64 + side * 32 + lane_off, s);
        tc::wait_ld();
        if (!(a.scale_log2 > 0.f)) {
#pragma unroll
          for (int c = 0; c < 32; ++c)
            s[c] = a.scale_log2 < 0.f ? s[c] ^ 0x80000000u : __float_as_uint(__uint_as_float(s[c]) * 0.f);
        }
        if (live < 32) {
#pragma unroll
          for (int c = 0; c < 32; ++c)
            if (c >= live) s[c] = 0xFF800000u;
        }
        if (j + 1 < sg.j1) live = live_of(sg, j + 1);
        float x[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 16; ++c)
          x[c & 1] = max3(x[c & 1], __uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1]));
        // two buffers: a warp may be at the next tile before the others have read this one's
        float* const sx = s_x + (t & 1) * 256;
        sx[tid] = fmaxf(x[0], x[1]);
        row_sync();
        const float mt = sc * fmaxf(fmaxf(sx[tid], sx[tid ^ 64]), fmaxf(sx[tid ^ 128], sx[tid ^ 192]));
        const bool up = mt > m + LD_TOP || (m == -INFINITY && mt > m);
        const float m_new = up ? mt : m;
        const float mm = m_new == -INFINITY ? 0.f : m_new;
        const uint64_t kk = f32x2(sc, sc), cc = f32x2(-mm, -mm);
        uint64_t sum = f32x2(0.f, 0.f);
        uint32_t p[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          float d0, d1;
          unpack_f32x2(fma_f32x2(f32x2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), kk, cc),
                       d0, d1);
          p[c] = pack_bf16x2(fast_exp2(d0), fast_exp2(d1));
          // of the rounded weights, so that they add up to one
          sum = add_f32x2(sum, f32x2(bf16lo_to_f32(p[c]), bf16hi_to_f32(p[c])));
        }
        if (j > sg.j0) {   // P is free, and O complete up to the last tile
          ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(pv_done, (t - 1) & 1)) != 0;
          if (__any_sync(0xffffffffu, up)) {
            tc::fence_after();
            const float f = up && m != -INFINITY ? fast_exp2(m - m_new) : 1.f;
#pragma unroll 1
            for (int c0 = side * (R / 4); c0 < (side + 1) * (R / 4); c0 += 32) {
              uint32_t o[32];
              tc::ld32(tO + c0 + lane_off, o);
              tc::wait_ld();
#pragma unroll
              for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
              tc::st32(tO + c0 + lane_off, o);
            }
            tc::wait_st();
            l *= f;
          }
        }
        const uint32_t to = sp + half * L::CHUNK + r * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          sts128(to + (((4 * side + k) ^ (r & 7)) << 4), p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]);
        fence_proxy_async_smem();
        tc::fence_before();
        __syncwarp();
        if (lane == 0 && ok) tc::arrive_cluster(p_ready, 0);
        m = m_new;
        float u, v;
        unpack_f32x2(sum, u, v);
        l += u + v;
      }
      more = later_seg(a, pl, run, nx);
      ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(pv_done, (t - 1) & 1)) != 0;
      tc::fence_after();
      float* const sx = s_x + (t & 1) * 256;
      sx[tid] = l;
      row_sync();
      l = (sx[tid] + sx[tid ^ 64]) + (sx[tid ^ 128] + sx[tid ^ 192]);
      const bool whole = sg.j1 - sg.j0 == sg.n;
      const bool direct = whole && a.num_groups == 0;
      const int64_t prow =
          whole ? (int64_t)2 * pl.pairs * pl.slot_rows +
                      (sg.item < pl.prefix_items ? 0 : (int64_t)a.batch * a.H) + sg.it.row0
                : (int64_t)(2 * pair + (sg.j0 == 0 ? 1 : 0)) * pl.slot_rows;
      const int64_t crow = (direct ? (int64_t)sg.it.row0 : prow) + 64 * rank;   // this CTA's first row
      const int rows = __all_sync(0xffffffffu, ok) ? sg.it.nrows - 64 * (int)rank : 0;
      if (!direct && half == 0 && side == 0 && r < rows)
        *reinterpret_cast<float2*>(pl.ml + (crow + r) * 2) = make_float2(m, l);
      const float inv = l != 0.f ? 1.f / l : 0.f;
      // O is read in pieces of 16 rows x 8 columns, of which four threads have 32 bytes of a row: whole
      // sectors are written from the registers.  (Through shared memory, a row a thread, this took
      // 1.4 us for 16 rows and 3 us for 64.)  A short loop for the instruction caches' sake: written out over
      // R / 4 columns, 4,096 requests of 64 positions x 16 heads took 290 us for 266.
      const int row_base = (quarter & 1) * 32, sub = lane >> 2, col = lane & 3;
#pragma unroll 1
      for (int r0 = row_base; r0 < min(row_base + 32, rows); r0 += 16) {
        const bool lo = r0 + sub < rows, hi = r0 + sub + 8 < rows;
        const uint32_t from = tO + lane_off + ((uint32_t)(r0 - row_base) << 16) + side * (R / 4);
        const float f0 = __shfl_sync(0xffffffffu, inv, r0 - row_base + sub);
        const float f1 = __shfl_sync(0xffffffffu, inv, r0 - row_base + sub + 8);
        // this thread's R / 4 columns adjoin in a row of O
        const int64_t at = (crow + r0 + sub) * R + half * 128 + (R == 512 ? side * 256 : side * 64);
#pragma unroll 1
        for (int c = 0; c < R / 4; c += 32) {
          uint32_t o[16];
          ld16_32(from + c, o);
          tc::wait_ld();
          if (direct) {   // neighbours exchange a piece: eight bytes each
            uint16_t* const to = a.out + at + c + 8 * (col & 1) + 4 * (col >> 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // pieces 0 and 1, then 2 and 3, of both rows
              const uint32_t* const x = o + 8 * (i >> 1) + 2 * (i & 1);
              const float f = i & 1 ? f1 : f0;
              const uint32_t u = pack_bf16x2(__uint_as_float(x[0]) * f, __uint_as_float(x[1]) * f);
              const uint32_t v = pack_bf16x2(__uint_as_float(x[4]) * f, __uint_as_float(x[5]) * f);
              const uint32_t w = __shfl_xor_sync(0xffffffffu, col & 1 ? u : v, 1);
              if (i & 1 ? hi : lo)
                *reinterpret_cast<uint2*>(to + 8 * R * (i & 1) + 16 * (i >> 1)) =
                    col & 1 ? make_uint2(w, v) : make_uint2(u, w);
            }
          } else {
            float* const to = pl.o + at + c + 2 * col;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (lo) *reinterpret_cast<uint2*>(to + 8 * i) = make_uint2(o[4 * i], o[4 * i + 1]);
              if (hi) *reinterpret_cast<uint2*>(to + 8 * R + 8 * i) = make_uint2(o[4 * i + 2], o[4 * i + 3]);
            }
          }
        }
      }
      tc::fence_before();
      sg = nx;
      row_sync();   // s_x read before a warp goes on to write it
    }
  }

  // Neither CTA may release TMEM or exit while its partner can still reach it.  CTA 1's arrivals (K, V, Q, P) were
  // all waited for by the products they belong to, the products' by copies and softmax.
  tc::fence_before();
  if (!settle(ok) && threadIdx.x == 0) flag_error(a.status, JF_DEV_ERR_TIMEOUT);
  cluster_meet();
  if (warp == 0) {
    tc::fence_after();
    tc::dealloc2(*tmem_slot, 512);
  }
}

// ---------------------------------------------------------------------------
// Join the partials of each row that has any.
// ---------------------------------------------------------------------------
constexpr int LM_THREADS = 256, LM_BATCH = 8, LM_WARPS = LM_THREADS / 32;
constexpr int LM_MAX = 256;   // partials of a row: at most 2 (pairs + 1)

// The rows of a row's partials over prefixes: those of the prefix's item, then its own's.
__device__ __forceinline__ int places_of(const LatentDecode& a, const LatentPlan& pl, uint32_t row, int lane,
                                         int32_t* rows) {
  const uint32_t total = (uint32_t)a.batch * (uint32_t)a.H;   // below 2^26
  const int b = (int)(row / (uint32_t)a.H), h = (int)(row - (uint32_t)b * (uint32_t)a.H);
  const int64_t units = *pl.units;
  int g = 0;
  while (a.first[g + 1] <= b) ++g;
  const int at = (int)(row - (uint32_t)a.first[g] * (uint32_t)a.H);
  const int2 span[2] = {pl.spans[pl.item0[g] + at / LD_ROWS],
                        pl.spans[pl.prefix_items + b * pl.blocks + h / LD_ROWS]};
  const int inside[2] = {at % LD_ROWS, h % LD_ROWS};
  const PairRuns runs(units, pl.pairs, pl.inv);
  int count = 0;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const int p0 = span[part].x, p1 = span[part].y;
    if (p1 < p0) continue;   // nothing there
    if (p0 == p1) {
      if (lane == 0)
        rows[count] = (int32_t)(2 * pl.pairs * pl.slot_rows + (part == 0 ? 0 : total) + row);
      ++count;
      continue;
    }
    for (int p = p0 + lane; p - lane <= p1; p += 32) {   // those that have units at all
      const bool has = p <= p1 && runs.first(p) < runs.first(p + 1);
      const unsigned m = __ballot_sync(0xffffffffu, has);
      if (has)
        rows[count + __popc(m & ((1u << lane) - 1))] =
            (2 * p + (p == p0 ? 1 : 0)) * pl.slot_rows + inside[part];
      count += __popc(m);
    }
  }
  __syncwarp();
  return count;
}

// Their weights, and one over the sum of all.
__device__ __forceinline__ float weights_of(const LatentPlan& pl, int count, int lane, const int32_t* rows,
                                            float2* w) {
  float M = -INFINITY, S = 0.f;
  for (int i = lane; i < count; i += 32) {
    w[i] = *reinterpret_cast<const float2*>(pl.ml + (int64_t)rows[i] * 2);
    M = fmaxf(M, w[i].x);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  for (int i = lane; i < count; i += 32) {
    // no maximum at all: sums of zero, or NaN where every score was
    const float f = M == -INFINITY ? 1.f : fast_exp2(w[i].x - M);
    S = fmaf(f, w[i].y, S);
    w[i].x = f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
  __syncwarp();
  return S != 0.f ? 1.f / S : 0.f;
}

__device__ __forceinline__ uint2 to_bf16(const float4& x, float f) {
  return make_uint2(pack_bf16x2(x.x * f, x.y * f), pack_bf16x2(x.z * f, x.w * f));
}

// A CTA takes CH channels of a row: first its partials' places and, a thread each, their weights; then a
// thread 4 channels, the partials in turn over the groups of CH / 4 threads, eight loads in flight.  (Places
// and weights by each warp on its own, as below, took one request of 131,072 positions x 128 heads 41.7 us
// for 40.6.)
template <int R, int CH>
__global__ void __launch_bounds__(LM_THREADS)
latent_merge_kernel(const __grid_constant__ LatentDecode a, const __grid_constant__ LatentPlan pl) {
  constexpr int LANES = CH / 4, GROUPS = LM_THREADS / LANES, WARPS = LM_WARPS;
  __shared__ float s_w[LM_THREADS];
  __shared__ int32_t s_row[LM_THREADS];
  __shared__ float s_red[2][WARPS];
  __shared__ int32_t s_cnt[WARPS];
  __shared__ float4 s_o[LM_THREADS];
  __shared__ uint32_t s_list[LM_THREADS];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = (int)threadIdx.x % LANES, grp = (int)threadIdx.x / LANES;
  const uint32_t total = (uint32_t)a.batch * (uint32_t)a.H, slices = total * (R / CH);   // below 2^28
  // More rows than blocks (of a decode, CH = R): a thread looks a row over, and the block takes those that are
  // not written out already.  (A block a row in turn, 4,096 requests of 64 positions x 16 heads took 266 us, 203 so.)
  const bool list = CH == R && gridDim.x < slices;
  for (uint32_t base = blockIdx.x; base < slices; base += gridDim.x * LM_THREADS) {
    int todo = 1;
    if (list) {
      const uint32_t mine = base + threadIdx.x * gridDim.x;
      bool need = false;
      if (mine < slices) {
        const uint32_t b = mine / (uint32_t)a.H, h = mine - b * (uint32_t)a.H;
        const int2 span = pl.spans[(int)b * pl.blocks + (int)h / LD_ROWS];
        need = span.x != span.y;
      }
      const unsigned m = __ballot_sync(0xffffffffu, need);
      if (lane == 0) s_cnt[warp] = __popc(m);
      __syncthreads();
      int at = 0;
      todo = 0;
      for (int w = 0; w < WARPS; ++w) {
        if (w < warp) at += s_cnt[w];
        todo += s_cnt[w];
      }
      if (need) s_list[at + __popc(m & ((1u << lane) - 1))] = mine;
      __syncthreads();
    }
    for (int t = 0; t < todo; ++t) {
      const uint32_t slice = list ? s_list[t] : base;
      const uint32_t row = slice / (R / CH);
      const int ch = (int)(slice % (R / CH)) * CH + c * 4;
      const int b = (int)(row / (uint32_t)a.H), h = (int)(row - (uint32_t)b * (uint32_t)a.H);
      // the row's partials: those of the prefix's item, then its own's
      const int64_t units = *pl.units;
      int count = 0;
      bool direct = false;
      for (int part = CH < R && a.num_groups ? 0 : 1; part < 2; ++part) {   // CH = R: no prefixes
        int item, inside;
        if (part == 0) {
          int g = 0;
          while (a.first[g + 1] <= b) ++g;
          inside = (int)(row - (uint32_t)a.first[g] * (uint32_t)a.H);
          item = pl.item0[g] + inside / LD_ROWS;
          inside %= LD_ROWS;
        } else {
          item = pl.prefix_items + b * pl.blocks + h / LD_ROWS;
          inside = h % LD_ROWS;
        }
        const int2 span = pl.spans[item];
        const int p0 = span.x, p1 = span.y;
        if (p1 < p0) continue;   // nothing there
        if (p0 == p1) {
          if (a.num_groups == 0) direct = true;
          if (threadIdx.x == 0)
            s_row[count] = (int32_t)(2 * pl.pairs * pl.slot_rows + (part == 0 ? 0 : total) + row);
          ++count;
          continue;
        }
        // pairs between the first and the last that have units at all
        const PairRuns runs(units, pl.pairs, pl.inv);
        const int p = p0 + (int)threadIdx.x;
        const bool has = p <= p1 && runs.first(p) < runs.first(p + 1);
        const unsigned m = __ballot_sync(0xffffffffu, has);
        if (lane == 0) s_cnt[warp] = __popc(m);
        __syncthreads();
        int at = count;
        for (int w = 0; w < WARPS; ++w) {
          if (w < warp) at += s_cnt[w];
          count += s_cnt[w];
        }
        if (has)
          s_row[at + __popc(m & ((1u << lane) - 1))] = (2 * p + (p == p0 ? 1 : 0)) * pl.slot_rows + inside;
        __syncthreads();
      }
      if (direct) continue;   // uniform over the CTA
      __syncthreads();
      // the first loads, under way while the weights are worked out
      const float* const src = pl.o + ch;
      float4 v[LM_BATCH];
#pragma unroll
      for (int k = 0; k < LM_BATCH; ++k)
        if (grp + k * GROUPS < count)
          v[k] = *reinterpret_cast<const float4*>(src + (int64_t)s_row[grp + k * GROUPS] * R);
      float m = -INFINITY, l = 0.f;
      if ((int)threadIdx.x < count) {
        const float2 x = *reinterpret_cast<const float2*>(pl.ml + (int64_t)s_row[threadIdx.x] * 2);
        m = x.x;
        l = x.y;
      }
      float M = m;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      if (lane == 0) s_red[0][warp] = M;
      __syncthreads();
      M = s_red[0][0];
      for (int w = 1; w < WARPS; ++w) M = fmaxf(M, s_red[0][w]);
      // no maximum at all: sums of zero, or NaN where every score was
      const float f = M == -INFINITY ? 1.f : fast_exp2(m - M);
      float S = f * l;
      s_w[threadIdx.x] = f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
      if (lane == 0) s_red[1][warp] = S;
      __syncthreads();
      S = 0.f;
      for (int w = 0; w < WARPS; ++w) S += s_red[1][w];
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = grp; i < count; i += LM_BATCH * GROUPS) {
#pragma unroll
        for (int k = 0; k < LM_BATCH; ++k)
          if (i + k * GROUPS < count) {
            const float w = s_w[i + k * GROUPS];
            acc.x = fmaf(v[k].x, w, acc.x);
            acc.y = fmaf(v[k].y, w, acc.y);
            acc.z = fmaf(v[k].z, w, acc.z);
            acc.w = fmaf(v[k].w, w, acc.w);
          }
        const int next = i + LM_BATCH * GROUPS;
#pragma unroll
        for (int k = 0; k < LM_BATCH; ++k)
          if (next + k * GROUPS < count)
            v[k] = *reinterpret_cast<const float4*>(src + (int64_t)s_row[next + k * GROUPS] * R);
      }
      s_o[threadIdx.x] = acc;
      __syncthreads();
      if (grp == 0) {
        for (int g = 1; g < GROUPS; ++g) {
          const float4 x = s_o[g * LANES + c];
          acc.x += x.x;
          acc.y += x.y;
          acc.z += x.z;
          acc.w += x.w;
        }
        const float inv = S != 0.f ? 1.f / S : 0.f;
        *reinterpret_cast<uint2*>(a.out + (int64_t)row * R + ch) = to_bf16(acc, inv);
      }
      __syncthreads();
    }
  }
}

// The same for many rows over prefixes, each with a pair's part or more to join: a warp 128 channels
// of a row, its places and weights worked out on its own.
template <int R>
__global__ void __launch_bounds__(LM_THREADS)
latent_merge_rows_kernel(const __grid_constant__ LatentDecode a, const __grid_constant__ LatentPlan pl) {
  __shared__ int32_t s_row[LM_WARPS][LM_MAX];
  __shared__ float2 s_w[LM_WARPS][LM_MAX];   // (m, l), then the weight
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t slice = blockIdx.x * LM_WARPS + warp, row = slice / (R / 128);
  const int ch = (int)(slice % (R / 128)) * 128 + lane * 4;
  if (row >= (uint32_t)a.batch * (uint32_t)a.H) return;
  int32_t* const rows = s_row[warp];
  float2* const w = s_w[warp];
  const int count = places_of(a, pl, row, lane, rows);
  const float* const src = pl.o + ch;
  float4 v[LM_BATCH];
  auto load = [&](int i) {
#pragma unroll
    for (int k = 0; k < LM_BATCH; ++k)
      if (i + k < count) v[k] = *reinterpret_cast<const float4*>(src + (int64_t)rows[i + k] * R);
  };
  load(0);   // under way while the weights are worked out
  const float inv = weights_of(pl, count, lane, rows, w);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < count; i += LM_BATCH) {
#pragma unroll
    for (int k = 0; k < LM_BATCH; ++k)
      if (i + k < count) {
        const float f = w[i + k].x;
        acc.x = fmaf(v[k].x, f, acc.x);
        acc.y = fmaf(v[k].y, f, acc.y);
        acc.z = fmaf(v[k].z, f, acc.z);
        acc.w = fmaf(v[k].w, f, acc.w);
      }
    load(i + LM_BATCH);
  }
  *reinterpret_cast<uint2*>(a.out + (int64_t)row * R + ch) = to_bf16(acc, inv);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// items, and the partials' rows
static void plan_sizes(int64_t batch, int64_t H, int64_t groups, int64_t sms, int64_t* items,
                       int64_t* slot_rows, int64_t* rows) {
  const int64_t pairs = sms / 2;
  // a group's rows fill ceil(rows / 128) items; at most one of them is partly filled
  *items = batch * ((H + LD_ROWS - 1) / LD_ROWS) + (groups ? groups + batch * H / LD_ROWS : 0);
  *slot_rows = groups || H > LD_ROWS ? LD_ROWS : H;
  *rows = 2 * pairs * *slot_rows + (groups ? 2 * batch * H : 0);
}

size_t latent_decode_workspace_bytes(int64_t batch, int64_t H, int64_t R, int64_t groups, int64_t sms) {
  int64_t items, slot_rows, rows;
  plan_sizes(batch, H, groups, sms, &items, &slot_rows, &rows);
  return (size_t)(256 + round256((items + 1) * 8) + round256(rows * 8) + rows * R * 4);
}

template <int R>
static int launch_t(const LatentDecode& a, const LatentPlan& pl, cudaStream_t stream) {
  // a copy brings 64 rows of several 64-channel chunks: issued one chunk a copy, a tile's K alone kept its
  // thread for 0.6 us
  CUtensorMap kmap, vmap, qmap;
  int st = bf16_chunks_map(a.pool.base, a.pool.row, a.pool.num_pages * a.pool.P, LdSmem<R>::KC, &kmap);
  if (!st) st = bf16_chunks_map(a.pool.base, a.pool.row, a.pool.num_pages * a.pool.P, 2, &vmap);
  if (!st) st = bf16_chunks_map(a.q, a.pool.row, (int64_t)a.batch * a.H, LdSmem<R>::KC, &qmap);
  if (st) return st;
  if (smem_optin((const void*)latent_decode_kernel<R>, LdSmem<R>::TOTAL) != JF_OK) return JF_ERR_CUDA;
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * (unsigned)pl.pairs);
  cfg.blockDim = dim3(LD_THREADS);
  cfg.dynamicSmemBytes = LdSmem<R>::TOTAL;
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, latent_decode_kernel<R>, kmap, vmap, qmap, a, pl) != cudaSuccess) return JF_ERR_CUDA;
  // Few rows: 128 channels a CTA, so that more of the GPU takes part (one request of 131,072 positions
  // x 128 heads 39.7 us, a CTA a row 43.7).  Many: a CTA a row, since most of a decode's rows have a few
  // parts or none (32 mixed requests 101.5 us, 128 channels a CTA 105.5); over prefixes a warp 128
  // channels (64 continuations 55.6 us, a CTA a row 57.3; 2 x 4 continuations x 128 heads 21.5 and 23.0).
  const int64_t rows = (int64_t)a.batch * a.H, slices = rows * (R / 128);
  const bool many = rows >= 4 * pl.pairs;
  cfg.blockDim = dim3(LM_THREADS);
  cfg.dynamicSmemBytes = 0;
  cudaError_t e;
  if (!many) {
    cfg.gridDim = dim3((unsigned)slices);
    e = cudaLaunchKernelEx(&cfg, latent_merge_kernel<R, 128>, a, pl);
  } else if (!a.num_groups) {
    cfg.gridDim = dim3((unsigned)(rows < 16 * pl.pairs ? rows : 16 * pl.pairs));
    e = cudaLaunchKernelEx(&cfg, latent_merge_kernel<R, R>, a, pl);
  } else {
    cfg.gridDim = dim3((unsigned)((slices + LM_WARPS - 1) / LM_WARPS));
    e = cudaLaunchKernelEx(&cfg, latent_merge_rows_kernel<R>, a, pl);
  }
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

int launch_latent_decode(const LatentDecode& a, void* workspace, cudaStream_t stream) {
  LatentPlan pl;
  int64_t items, slot_rows, rows;
  const int sms = sm_count();
  if (sms / 2 > LM_MAX / 2 - 2) return JF_ERR_UNSUPPORTED;
  plan_sizes(a.batch, a.H, a.num_groups, sms, &items, &slot_rows, &rows);
  uint8_t* ws = static_cast<uint8_t*>(workspace) + 256;
  pl.pairs = sms / 2;
  pl.inv = pairs_inverse(pl.pairs);
  pl.slot_rows = (int32_t)slot_rows;
  pl.blocks = (a.H + LD_ROWS - 1) / LD_ROWS;
  pl.item0[0] = 0;
  for (int g = 0; g < a.num_groups; ++g)
    pl.item0[g + 1] = pl.item0[g] + ((a.first[g + 1] - a.first[g]) * a.H + LD_ROWS - 1) / LD_ROWS;
  pl.prefix_items = a.num_groups ? pl.item0[a.num_groups] : 0;
  pl.items = pl.prefix_items + a.batch * pl.blocks;
  pl.units = reinterpret_cast<int64_t*>(ws);
  pl.spans = reinterpret_cast<int2*>(ws) + 1;
  ws += round256((items + 1) * 8);
  pl.ml = reinterpret_cast<float*>(ws);
  ws += round256(rows * 8);
  pl.o = reinterpret_cast<float*>(ws);
  return a.pool.R == 512 ? launch_t<512>(a, pl, stream) : launch_t<256>(a, pl, stream);
}

}  // namespace jfkv
