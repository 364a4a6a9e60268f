// Eviction from the 8-bit cache by accumulated attention weight.
//
// Select kernel: which positions of a (request, KV head) stay.  The first
// `sinks` and the last `recent` positions always do; of the others those with
// the largest weights, equal weights in order of position.  Weights map to
// 32-bit keys whose unsigned order is theirs (a protected position takes the
// largest key, NaN the smallest).  A cluster of up to 16 CTAs shares a row: each
// keeps the keys of its range of positions in shared memory, read from memory
// once, and a radix select over the cluster's histograms (11, 11 and 10 bits,
// added up through distributed shared memory) finds the budget-th largest
// key.  The kept positions are then written in rising order: all above that
// key, and the first of those that equal it.
//
// Compact kernel: a CTA gathers 32 kept positions of one KV head and writes them
// as one block, K and V, of the destination pages.  The block gets the
// scale its own rows call for; a row whose old scale differs is rounded again
// under it (an exact shift but for what falls below the smallest code).
//
// Bound: the select kernel by its chain of steps (load, three digits with an exchange
// each, count, pack), the compact kernel by memory.  One request of 262,144 positions,
// 4 KV heads x 256, cut to 32,768: select 20 us (4 MB of weights), compact 25 us
// (136 MB, 5.4 TB/s); 8 requests of up to 16,383 cut to 2,048 (D = 128): 13 and 10 us.
#include "kv8.cuh"

namespace jfkv {

constexpr int EV_THREADS = 1024;
constexpr int EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;
constexpr int EV_SLICE = 4096;              // keys a CTA should have before a row takes more CTAs
constexpr int EV_MAX_CLUSTER = 16;
constexpr int EV_MAX_KEYS = 48 * 1024;      // keys that fit a CTA's shared memory

struct EvictArgs {
  uint8_t* pool;
  int64_t num_pages;
  int64_t page_bytes;
  int64_t codes_region;
  int64_t sb_region;
  int32_t P, log2P, Hkv, B;
  const int32_t* page_table;
  int32_t pt_stride;
  const int32_t* ctx;
  const float* weights;        // [B, Hkv, wstride]
  int64_t wstride;
  int32_t budget, sinks, recent;
  const int32_t* dst_table;    // [B, dst_stride]
  int32_t dst_stride;
  int32_t* dst_ctx;            // [B]
  float* dst_weights;          // [B, Hkv, budget] or null
  int32_t* kept;               // [B, Hkv, budget]
  int32_t* err;
};

// Context of request b; 0 (and flagged by the select kernel) where it does not
// fit the page table or the weights.
__device__ __forceinline__ int ev_ctx(const EvictArgs& a, int b) {
  const int64_t c = a.ctx[b];
  return c < 0 || c > (int64_t)a.pt_stride * a.P || c > a.wstride ? 0 : (int)c;
}

// unsigned order = order of the weights; NaN, 1, below all of them, -0 as +0.
// 0 stands for no position: it is never kept.
__device__ __forceinline__ uint32_t ev_key(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 1u;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t ev_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t ev_ranks() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ void ev_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n"
               "barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
// this CTA's shared address `addr` in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t ev_map(uint32_t addr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(a) : "r"(addr), "r"(rank));
  return a;
}
__device__ __forceinline__ int2 ev_remote2(uint32_t addr, uint32_t rank) {
  int2 v;
  asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];\n"
               : "=r"(v.x), "=r"(v.y) : "r"(ev_map(addr, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void ev_remote_add(uint32_t addr, uint32_t rank, int v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.s32 [%0], %1;\n"
               ::"r"(ev_map(addr, rank)), "r"(v) : "memory");
}

// One count per key with `in` set, at once for a warp whose keys share a bin
// (weights that are all alike).  Whole warps.
__device__ __forceinline__ void ev_count(int* hist, uint32_t bin, bool in, int lane) {
  const uint32_t lead = __shfl_sync(0xffffffffu, bin, 0);
  if (__all_sync(0xffffffffu, in && bin == lead)) {
    if (lane == 0) atomicAdd(&hist[bin], 32);
  } else if (in) {
    atomicAdd(&hist[bin], 1);
  }
}

// CACHED: a CTA's keys fit its shared memory (rows up to 16 x 48 Ki positions);
// otherwise they are made again from the weights wherever they are needed.
template <bool CACHED>
__global__ void __launch_bounds__(EV_THREADS, 1) kv8_select_kernel(const EvictArgs a) {
  extern __shared__ __align__(16) uint32_t keys[];   // this CTA's slice
  __shared__ __align__(8) int hist[3][EV_BINS];      // one a digit
  __shared__ int sums[2][EV_WARPS];
  __shared__ int pick[2];
  __shared__ __align__(8) int mine[2];      // keys above, and equal to, the last one kept
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const uint32_t rank = ev_rank(), ranks = ev_ranks();
  const int h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = ev_ctx(a, b);
  if (h == 0 && rank == 0 && tid == 0) {
    if (n != a.ctx[b]) flag_error(a.err, JF_DEV_ERR_POSITION);
    a.dst_ctx[b] = min(n, a.budget);
  }
  const int64_t row = (int64_t)b * a.Hkv + h;
  const float* const w = a.weights + row * a.wstride;
  int32_t* const kept = a.kept + row * a.budget;
  float* const wout = a.dst_weights ? a.dst_weights + row * a.budget : nullptr;
  if (n <= a.budget) {   // everything stays (the whole cluster takes this way)
    for (int j = rank * EV_THREADS + tid; j < a.budget; j += ranks * EV_THREADS) {
      kept[j] = j < n ? j : -1;
      if (wout) wout[j] = j < n ? w[j] : 0.f;
    }
    return;
  }
  // this CTA's positions [p0, p0 + len), len a multiple of 128; those below 0 or from
  // n on are none.  Ranges start where a 16-byte load of the weights may.
  const int skew = (int)((reinterpret_cast<uintptr_t>(w) >> 2) & 3);
  const int64_t all = (int64_t)n + skew;
  const int slice = (int)((all + 128 * (int64_t)ranks - 1) / (128 * (int64_t)ranks)) * 128;
  const int64_t first = min((int64_t)rank * slice, all);
  const int p0 = (int)(first - skew);
  const int len = (int)min((int64_t)slice, (all - first + 127) / 128 * 128);
  auto key_at = [&](int i, float x) -> uint32_t {   // of position p0 + i with weight x
    const int t = p0 + i;
    if (t < 0 || t >= n) return 0u;
    return t < a.sinks || t >= n - a.recent ? 0xFFFFFFFFu : ev_key(x);
  };
  auto key1 = [&](int i) -> uint32_t {
    if (CACHED) return keys[i];
    const int t = p0 + i;
    return t >= 0 && t < n ? key_at(i, w[t]) : 0u;
  };
  auto key4 = [&](int i) -> uint4 {
    if (CACHED) return *reinterpret_cast<const uint4*>(keys + i);
    return make_uint4(key1(i), key1(i + 1), key1(i + 2), key1(i + 3));
  };
  for (int i = tid; i < 3 * EV_BINS; i += EV_THREADS) hist[0][i] = 0;
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");   // zeroed
  if (CACHED) {   // four 16-byte loads in flight a thread (16 of 4 bytes: 84.6 us, not 80.5)
    constexpr int U = 4;
    for (int ib = 4 * tid; ib < len; ib += 4 * U * EV_THREADS) {
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = ib + 4 * u * EV_THREADS, t = p0 + i;
        x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < len && t >= 0 && t < n - 3) {
          x[u] = *reinterpret_cast<const float4*>(w + t);
        } else if (i < len) {   // a row's ends
          if (t >= 0 && t < n) x[u].x = w[t];
          if (t >= -1 && t < n - 1) x[u].y = w[t + 1];
          if (t >= -2 && t < n - 2) x[u].z = w[t + 2];
          if (t >= -3 && t < n - 3) x[u].w = w[t + 3];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = ib + 4 * u * EV_THREADS;
        if (i < len)
          *reinterpret_cast<uint4*>(keys + i) =
              make_uint4(key_at(i, x[u].x), key_at(i + 1, x[u].y), key_at(i + 2, x[u].z),
                         key_at(i + 3, x[u].w));
      }
    }
  }
  __syncthreads();
  // the budget-th largest key, digit by digit from the top
  uint32_t prefix = 0;
  int need = a.budget;   // how many of the keys with this prefix stay
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int bits = pass == 2 ? 10 : 11;
    const uint32_t mask = (1u << bits) - 1u;
    int* const hs = hist[pass];
#pragma unroll 2
    for (int ib = 128 * warp; ib < len; ib += 128 * EV_WARPS) {   // whole warps take part
      const uint4 k4 = key4(ib + 4 * lane);
      const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
      bool in[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) in[i] = pass == 0 || (k[i] >> (shift + bits)) == prefix;
      // after the first digit few keys are left
      if (pass > 0 && !__any_sync(0xffffffffu, in[0] || in[1] || in[2] || in[3])) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) ev_count(hs, (k[i] >> shift) & mask, in[i], lane);
    }
    __syncthreads();
    if (pass == 0) asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    // Each CTA gathers the cluster's counts of its share of the bins: the others
    // add theirs to it, most bins being empty (reading all of every CTA's
    // histogram took 12,000 cycles of a 16-CTA cluster).
    const int share = (1 << bits) / (int)ranks;   // bins per CTA, even
    if (ranks > 1) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int bin = tid + u * EV_THREADS;
        if (bin <= (int)mask && bin / share != (int)rank) {
          const int c = hs[bin];
          if (c) ev_remote_add(smem_u32(hs + bin), bin / share, c);
        }
      }
      ev_cluster_sync();
    }
    // thread i looks at bins top - 2i and top - 2i - 1; the largest digit with
    // at least `need` keys at or above it is picked
    const int top = (int)mask;
    int c0 = 0, c1 = 0;
    if (2 * tid <= top) {
      const int bin = top - 2 * tid - 1;
      const int2 v = ranks > 1 ? ev_remote2(smem_u32(hs + bin), bin / share)
                               : *reinterpret_cast<const int2*>(hs + bin);
      c0 = v.y;
      c1 = v.x;
    }
    int incl = c0 + c1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) sums[0][warp] = incl;
    __syncthreads();
    const int above =
        __reduce_add_sync(0xffffffffu, lane < warp ? sums[0][lane] : 0) + incl - c0 - c1;
    if (above < need && need <= above + c0) {
      pick[0] = top - 2 * tid;
      pick[1] = need - above;
    } else if (above + c0 < need && need <= above + c0 + c1) {
      pick[0] = top - 2 * tid - 1;
      pick[1] = need - above - c0;
    }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)pick[0];
    need = pick[1];
    __syncthreads();
  }
  // ordered compaction: each warp a contiguous range [i0, i1) of the CTA's keys
  const int per = ((len + EV_WARPS - 1) / EV_WARPS + 127) & ~127;
  const int i0 = min(warp * per, len), i1 = min(i0 + per, len);
  int above = 0, equal = 0;
#pragma unroll 2
  for (int i = i0 + 4 * lane; i < i1; i += 128) {
    const uint4 k = key4(i);
    above += (k.x > prefix) + (k.y > prefix) + (k.z > prefix) + (k.w > prefix);
    equal += (k.x == prefix) + (k.y == prefix) + (k.z == prefix) + (k.w == prefix);
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    sums[0][warp] = above;
    sums[1][warp] = equal;
  }
  __syncthreads();
  int at, eq;   // keys above, and equal, before this warp's range
  {
    const int x = sums[0][lane], y = sums[1][lane];
    at = __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
    eq = __reduce_add_sync(0xffffffffu, lane < warp ? y : 0);
    if (warp == 0) {
      const int xs = __reduce_add_sync(0xffffffffu, x), ys = __reduce_add_sync(0xffffffffu, y);
      if (lane == 0) {
        mine[0] = xs;
        mine[1] = ys;
      }
    }
  }
  ev_cluster_sync();
  if (rank > 0) {
    const int2 v = lane < (int)rank ? ev_remote2(smem_u32(mine), lane) : make_int2(0, 0);
    at += __reduce_add_sync(0xffffffffu, v.x);
    eq += __reduce_add_sync(0xffffffffu, v.y);
  }
  // No CTA leaves while another may read its counts: this one's reads are done, at and
  // eq being made of them.  Nothing else is published, so nothing is waited for here.
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n" ::"r"(at), "r"(eq) : "memory");
  // A warp first packs its kept positions over its own range of the keys (no
  // more are kept than have been read), then writes them out in whole lines.
  const unsigned lower = (1u << lane) - 1u;
  const int jw = at + min(eq, need);   // this warp's first place
  int j = jw;
  auto put = [&](int to, int t) {
    if (CACHED) keys[i0 + to - jw] = (uint32_t)t;
    else kept[to] = t;
  };
  for (int ib = i0; ib < i1; ib += 128) {
    uint32_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = key1(ib + 32 * i + lane);
    const bool same = k[0] == prefix || k[1] == prefix || k[2] == prefix || k[3] == prefix;
    if (__any_sync(0xffffffffu, same)) {   // rare, but for weights that are all alike
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned me = __ballot_sync(0xffffffffu, k[i] == prefix);
        const bool keep = k[i] > prefix || (k[i] == prefix && eq + __popc(me & lower) < need);
        const unsigned mk = __ballot_sync(0xffffffffu, keep);
        if (keep) put(j + __popc(mk & lower), p0 + ib + 32 * i + lane);
        j += __popc(mk);
        eq += __popc(me);
      }
    } else {
      unsigned mk[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) mk[i] = __ballot_sync(0xffffffffu, k[i] > prefix);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (k[i] > prefix) put(j + __popc(mk[i] & lower), p0 + ib + 32 * i + lane);
        j += __popc(mk[i]);
      }
    }
  }
  __syncwarp();
#pragma unroll 4
  for (int jj = jw + lane; jj < j; jj += 32) {
    const int t = CACHED ? (int)keys[i0 + jj - jw] : kept[jj];
    if (CACHED) kept[jj] = t;
    if (wout) wout[jj] = w[t];
  }
  __syncwarp();
  asm volatile("barrier.cluster.wait.aligned;\n" ::: "memory");
}

// Largest code of 16, signs apart (0x7F where a NaN is among them).
__device__ __forceinline__ uint32_t ev_top(uint4 w) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __vmaxu2(m, __vmaxu2(ws[i] & 0x7F007F00u, (ws[i] << 8) & 0x7F007F00u));
  return max(m >> 24, (m >> 8) & 0x7Fu);
}
// The same with NaN passed over.
__device__ __noinline__ uint32_t ev_top_finite(uint4 w) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  uint32_t m = 0;
  for (int i = 0; i < 16; ++i) {
    const uint32_t c = (ws[i >> 2] >> (8 * (i & 3))) & 0x7Fu;
    if (c != 0x7Fu) m = max(m, c);
  }
  return m;
}

template <int D>
__global__ void __launch_bounds__(256) kv8_compact_kernel(const EvictArgs a) {
  constexpr int LPR = D / 16;              // lanes per row, 16 codes each
  constexpr int RPP = 256 / LPR;           // rows per pass
  constexpr int NP = KV8_BLOCK / RPP;
  __shared__ float warp_max[2][8];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int h = blockIdx.y, b = blockIdx.z;
  const int j0 = blockIdx.x * KV8_BLOCK;
  const int li = threadIdx.x % LPR, rr = threadIdx.x / LPR;
  const int32_t* const kept = a.kept + ((int64_t)b * a.Hkv + h) * a.budget;
  // the kept positions, -1 past them, are loaded beside the context they depend on
  int kept_t[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = j0 + p * RPP + rr;
    kept_t[p] = j < a.budget ? kept[j] : -1;
  }
  const int m = min(ev_ctx(a, b), a.budget);
  if (j0 >= m) return;
  const int pd = j0 >> a.log2P, slot0 = j0 & (a.P - 1);
  const int32_t dst = pd < a.dst_stride ? a.dst_table[(int64_t)b * a.dst_stride + pd] : -1;
  uint4 x[NP][2];
  float s_old[NP][2];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = j0 + p * RPP + rr;
    x[p][0] = x[p][1] = make_uint4(0u, 0u, 0u, 0u);
    s_old[p][0] = s_old[p][1] = 0.f;
    if (j < m) {
      const int t = kept_t[p];
      const int32_t page = a.page_table[(int64_t)b * a.pt_stride + (t >> a.log2P)];
      if (page < 0 || page >= a.num_pages) {
        if (li == 0) flag_error(a.err, JF_DEV_ERR_PAGE_ID);   // the row becomes zeros
      } else {
        const int slot = t & (a.P - 1);
        const uint8_t* const rec = a.pool + (int64_t)page * a.page_bytes;
        const uint8_t* const code = rec + (int64_t)(h * a.P + slot) * D + li * 16;
        const uint8_t* const scale =
            rec + 2 * a.codes_region + (h * (a.P / KV8_BLOCK) + slot / KV8_BLOCK) * 4;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
          x[p][kind] = *reinterpret_cast<const uint4*>(code + kind * a.codes_region);
          s_old[p][kind] = *reinterpret_cast<const float*>(scale + kind * a.sb_region);
        }
      }
    }
  }
  // the block's largest finite magnitude: that of a thread's codes as whole numbers
  // (their order is the values'), then with the rows' scales
  uint32_t mag[NP][2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    float amax = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const uint4 w = x[p][kind];
      mag[p][kind] = ev_top(w);
      uint32_t top = mag[p][kind], lo, hi;
      if (top == 0x7Fu) top = ev_top_finite(w);
      f16x4_of_e4m3(top, lo, hi);
      amax = fmaxf(amax, f32x2_of_f16x2(lo).x * two8(exp8_of_scale(s_old[p][kind])));
    }
    // magnitudes: the order of their bits is theirs
    const uint32_t all = __reduce_max_sync(0xffffffffu, __float_as_uint(amax));
    if (lane == 0) warp_max[kind][warp] = __uint_as_float(all);
  }
  __syncthreads();
  if (dst < 0 || dst >= a.num_pages) {
    if (threadIdx.x == 0)
      flag_error(a.err, pd < a.dst_stride ? JF_DEV_ERR_PAGE_ID : JF_DEV_ERR_POSITION);
    return;
  }
  uint8_t* const rec = a.pool + (int64_t)dst * a.page_bytes;
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, warp_max[kind][i]);
    const int e = exp8_of(top);
    if (threadIdx.x == 0)
      *reinterpret_cast<float*>(rec + 2 * a.codes_region + kind * a.sb_region +
                                (h * (a.P / KV8_BLOCK) + slot0 / KV8_BLOCK) * 4) = two8(e);
    uint8_t* const codes =
        rec + kind * a.codes_region + (int64_t)(h * a.P + slot0) * D + li * 16;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int row = p * RPP + rr;
      if (j0 + row < m) {
        // a row under its own scale keeps its codes (NaN apart, which has one code)
        const int s = exp8_of_scale(s_old[p][kind]) - e;
        uint4 w = x[p][kind];
        if (s != 0 || mag[p][kind] == 0x7Fu)
          w = make_uint4(rescale_e4m3x4(w.x, s), rescale_e4m3x4(w.y, s), rescale_e4m3x4(w.z, s),
                         rescale_e4m3x4(w.w, s));
        *reinterpret_cast<uint4*>(codes + row * D) = w;
      }
    }
  }
}

int launch_kv8_evict(const Geom& g, const jf_kv_pool& pool, const int32_t* page_table,
                     int32_t pt_stride, const int32_t* ctx, int32_t batch, const float* weights,
                     int64_t wstride, int32_t budget, int32_t sinks, int32_t recent,
                     const int32_t* dst_table, int32_t dst_stride, int32_t* dst_ctx,
                     float* dst_weights, int32_t* kept, int32_t* err, cudaStream_t stream) {
  EvictArgs a;
  a.pool = static_cast<uint8_t*>(pool.base);
  a.num_pages = g.num_pages;
  a.page_bytes = g.page_bytes;
  a.codes_region = g.codes_region;
  a.sb_region = g.sb_region;
  a.P = g.P;
  a.log2P = __builtin_ctz((unsigned)g.P);
  a.Hkv = g.Hkv;
  a.B = batch;
  a.page_table = page_table;
  a.pt_stride = pt_stride;
  a.ctx = ctx;
  a.weights = weights;
  a.wstride = wstride;
  a.budget = budget;
  a.sinks = sinks;
  a.recent = recent;
  a.dst_table = dst_table;
  a.dst_stride = dst_stride;
  a.dst_ctx = dst_ctx;
  a.dst_weights = dst_weights;
  a.kept = kept;
  a.err = err;
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  // CTAs per row: one for each EV_SLICE keys of the longest row there may be, in
  // powers of two (8 requests of up to 16,383 positions, 4 KV heads, with 2,048, 4,096
  // and 8,192 keys a CTA: 39.2, 30.0 and 31.6 us with the read back; at 2,048 the CTAs,
  // one to an SM, no longer fit at once)
  int cl = 1;
  while (cl < EV_MAX_CLUSTER && wstride > (int64_t)cl * EV_SLICE) cl *= 2;
  const int64_t keys = (wstride + 3 + 128 * cl - 1) / (128 * cl) * 128;   // 3: the ranges' skew
  const bool cached = keys <= EV_MAX_KEYS;
  const void* const select = cached ? (const void*)kv8_select_kernel<true>
                                    : (const void*)kv8_select_kernel<false>;
  if (cached && smem_optin(select, EV_MAX_KEYS * 4) != JF_OK) return JF_ERR_CUDA;
  // clusters past 8 CTAs are opted into (a flag of the function: setting it again
  // changes nothing)
  if (cl > 8 &&
      cudaFuncSetAttribute(select, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
    return JF_ERR_CUDA;
  cudaLaunchAttribute attrs[2];
  attrs[0] = pdl[0];
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = (unsigned)cl;
  attrs[1].val.clusterDim.y = 1;
  attrs[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)cl, (unsigned)g.Hkv, (unsigned)batch);
  cfg.blockDim = dim3(EV_THREADS);
  cfg.dynamicSmemBytes = cached ? (size_t)keys * 4 : 0;
  cfg.stream = stream;
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  const cudaError_t es = cached ? cudaLaunchKernelEx(&cfg, kv8_select_kernel<true>, a)
                                : cudaLaunchKernelEx(&cfg, kv8_select_kernel<false>, a);
  if (es != cudaSuccess) return JF_ERR_CUDA;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  cfg.dynamicSmemBytes = 0;
  cfg.gridDim = dim3((unsigned)(((int64_t)budget + KV8_BLOCK - 1) / KV8_BLOCK), (unsigned)g.Hkv,
                     (unsigned)batch);
  cfg.blockDim = dim3(256);
  const cudaError_t e = g.D == 256 ? cudaLaunchKernelEx(&cfg, kv8_compact_kernel<256>, a)
                                   : cudaLaunchKernelEx(&cfg, kv8_compact_kernel<128>, a);
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv
