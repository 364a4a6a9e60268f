// Eviction from the 8-bit cache by accumulated attention weight.
//
// Select kernel: which positions of a (request, KV head) stay.  The first
// `sinks` and the last `recent` positions always do; of the others those with
// the largest weights, equal weights in order of position.  Weights map to
// 32-bit keys whose unsigned order is theirs (a protected position takes the
// largest key, NaN the smallest); a radix select finds the budget-th largest
// key 8 bits at a time, and the kept positions are then written in rising
// order: all above that key, and the first of those that equal it.
//
// Compact kernel: a CTA gathers 32 kept positions of one KV head, K or V, and
// writes them as one block of the destination pages.  The block gets the
// scale its own rows call for; a row whose old scale differs is rounded again
// under it (an exact shift but for what falls below the smallest code).
#include "kv8.cuh"

namespace jfkv {

constexpr int EV_THREADS = 1024;
constexpr int EV_WARPS = EV_THREADS / 32;

struct EvictArgs {
  uint8_t* pool;
  int64_t num_pages;
  int64_t page_bytes;
  int64_t codes_region;
  int64_t sb_region;
  int32_t P, Hkv, B;
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

// unsigned order = order of the weights; NaN below all, -0 as +0
__device__ __forceinline__ uint32_t ev_key(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0u;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(EV_THREADS, 1) kv8_select_kernel(const EvictArgs a) {
  __shared__ int hist[256];
  __shared__ int sums[2][EV_WARPS];
  __shared__ int pick[2];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int h = blockIdx.x, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = ev_ctx(a, b);
  if (h == 0 && tid == 0) {
    if (n != a.ctx[b]) flag_error(a.err, JF_DEV_ERR_POSITION);
    a.dst_ctx[b] = min(n, a.budget);
  }
  const int64_t row = (int64_t)b * a.Hkv + h;
  const float* const w = a.weights + row * a.wstride;
  int32_t* const kept = a.kept + row * a.budget;
  float* const wout = a.dst_weights ? a.dst_weights + row * a.budget : nullptr;
  if (n <= a.budget) {   // everything stays
    for (int j = tid; j < a.budget; j += EV_THREADS) {
      kept[j] = j < n ? j : -1;
      if (wout) wout[j] = j < n ? w[j] : 0.f;
    }
    return;
  }
  auto key_of = [&](int t) -> uint32_t {
    return t < a.sinks || t >= n - a.recent ? 0xFFFFFFFFu : ev_key(w[t]);
  };
  // the budget-th largest key, a byte at a time from the top
  uint32_t prefix = 0;
  int need = a.budget;   // how many of the keys with this prefix stay
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int t = tid; t < n; t += EV_THREADS) {
      const uint32_t k = key_of(t);
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (warp == 0) {   // the largest digit with at least `need` keys at or above it
      int s = 0;       // keys of this lane's 8 digits, from the top down
      for (int i = 0; i < 8; ++i) s += hist[255 - (8 * lane + i)];
      int incl = s;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      int above = incl - s;
      if (above < need && need <= incl) {
        for (int i = 0; i < 8; ++i) {
          const int d = 255 - (8 * lane + i);
          if (need <= above + hist[d]) {
            pick[0] = d;
            pick[1] = need - above;
            break;
          }
          above += hist[d];
        }
      }
    }
    __syncthreads();
    prefix = (prefix << 8) | (uint32_t)pick[0];
    need = pick[1];
    __syncthreads();
  }
  // ordered compaction: each warp a contiguous range of positions
  const int per = ((n + EV_WARPS - 1) / EV_WARPS + 31) & ~31;
  const int t0 = min(warp * per, n), t1 = min(t0 + per, n);
  int above = 0, equal = 0;
  for (int t = t0 + lane; t < t1; t += 32) {
    const uint32_t k = key_of(t);
    above += k > prefix;
    equal += k == prefix;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    above += __shfl_xor_sync(0xffffffffu, above, o);
    equal += __shfl_xor_sync(0xffffffffu, equal, o);
  }
  if (lane == 0) {
    sums[0][warp] = above;
    sums[1][warp] = equal;
  }
  __syncthreads();
  int eq = 0, at = 0;   // equal keys, and kept positions, before this warp's range
  for (int i = 0; i < warp; ++i) {
    at += sums[0][i];
    eq += sums[1][i];
  }
  at += min(eq, need);
  for (int tb = t0; tb < t1; tb += 32) {
    const int t = tb + lane;
    const uint32_t k = t < t1 ? key_of(t) : 0u;
    const unsigned mine = (1u << lane) - 1u;
    const unsigned me = __ballot_sync(0xffffffffu, t < t1 && k == prefix);
    const bool keep = t < t1 && (k > prefix || (k == prefix && eq + __popc(me & mine) < need));
    const unsigned mk = __ballot_sync(0xffffffffu, keep);
    if (keep) {
      const int j = at + __popc(mk & mine);
      kept[j] = t;
      if (wout) wout[j] = w[t];
    }
    at += __popc(mk);
    eq += __popc(me);
  }
}

template <int D>
__global__ void __launch_bounds__(256) kv8_compact_kernel(const EvictArgs a) {
  constexpr int LPR = D / 16;              // lanes per row, 16 codes each
  constexpr int RPP = 256 / LPR;           // rows per pass
  constexpr int NP = KV8_BLOCK / RPP;
  __shared__ float warp_max[8];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int h = blockIdx.y % a.Hkv, kind = blockIdx.y / a.Hkv, b = blockIdx.z;
  const int m = min(ev_ctx(a, b), a.budget);
  const int j0 = blockIdx.x * KV8_BLOCK;
  if (j0 >= m) return;
  const int li = threadIdx.x % LPR, rr = threadIdx.x / LPR;
  const int32_t* const kept = a.kept + ((int64_t)b * a.Hkv + h) * a.budget;
  uint4 x[NP];
  int e_old[NP];
  float amax = 0.f;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = j0 + p * RPP + rr;
    x[p] = make_uint4(0u, 0u, 0u, 0u);
    e_old[p] = KV8_EMIN;
    if (j < m) {
      const int t = kept[j];
      const int32_t page = a.page_table[(int64_t)b * a.pt_stride + t / a.P];
      if (page < 0 || page >= a.num_pages) {
        if (li == 0) flag_error(a.err, JF_DEV_ERR_PAGE_ID);   // the row becomes zeros
      } else {
        const int slot = t % a.P;
        const uint8_t* const rec = a.pool + (int64_t)page * a.page_bytes;
        x[p] = *reinterpret_cast<const uint4*>(rec + kind * a.codes_region +
                                               ((int64_t)h * a.P + slot) * D + li * 16);
        e_old[p] = exp8_of_scale(
            *(reinterpret_cast<const float*>(rec + 2 * a.codes_region + kind * a.sb_region) +
              h * (a.P / KV8_BLOCK) + slot / KV8_BLOCK));
      }
    }
    const uint32_t w[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
    uint32_t top = 0;   // largest finite magnitude code (its order is that of the values)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t c = (w[i] >> (8 * k)) & 0x7Fu;
        if (c != 0x7Fu) top = max(top, c);
      }
    uint32_t lo, hi;
    f16x4_of_e4m3(top, lo, hi);
    amax = fmaxf(amax, f32x2_of_f16x2(lo).x * two8(e_old[p]));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (lane == 0) warp_max[warp] = amax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, warp_max[i]);
  const int e = exp8_of(amax);
  const int32_t page = j0 / a.P < a.dst_stride ? a.dst_table[(int64_t)b * a.dst_stride + j0 / a.P] : -1;
  if (page < 0 || page >= a.num_pages) {
    if (threadIdx.x == 0)
      flag_error(a.err, j0 / a.P < a.dst_stride ? JF_DEV_ERR_PAGE_ID : JF_DEV_ERR_POSITION);
    return;
  }
  uint8_t* const rec = a.pool + (int64_t)page * a.page_bytes;
  uint8_t* const codes = rec + kind * a.codes_region + ((int64_t)h * a.P + j0 % a.P) * D;
  if (threadIdx.x == 0)
    *(reinterpret_cast<float*>(rec + 2 * a.codes_region + kind * a.sb_region) +
      h * (a.P / KV8_BLOCK) + (j0 % a.P) / KV8_BLOCK) = two8(e);
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int row = p * RPP + rr;
    if (j0 + row < m) {
      uint4 c = x[p];
      if (e_old[p] != e) {
        const float s = two8(e_old[p] - e);
        c.x = rescale_e4m3x4(c.x, s);
        c.y = rescale_e4m3x4(c.y, s);
        c.z = rescale_e4m3x4(c.z, s);
        c.w = rescale_e4m3x4(c.w, s);
      }
      *reinterpret_cast<uint4*>(codes + row * D + li * 16) = c;
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
  cfg.gridDim = dim3((unsigned)g.Hkv, (unsigned)batch);
  cfg.blockDim = dim3(EV_THREADS);
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kv8_select_kernel, a) != cudaSuccess) return JF_ERR_CUDA;
  cfg.gridDim = dim3((unsigned)((budget + KV8_BLOCK - 1) / KV8_BLOCK), (unsigned)(2 * g.Hkv),
                     (unsigned)batch);
  cfg.blockDim = dim3(256);
  const cudaError_t e = g.D == 256 ? cudaLaunchKernelEx(&cfg, kv8_compact_kernel<256>, a)
                                   : cudaLaunchKernelEx(&cfg, kv8_compact_kernel<128>, a);
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv
