// Append to and read back from the 8-bit block-scaled cache.
//
// Append.  The rows of request b (row_offsets[b] .. row_offsets[b + 1]) go to
// consecutive positions from start_pos[b].  A CTA takes one block of 32
// positions of one KV head, K or V: it holds the block's new rows in
// registers (32 rows x D bf16 over 256 threads), takes their largest
// magnitude, settles the block's exponent and writes the codes.  A block
// that already holds positions keeps the larger of its exponent and the new
// rows'; when it grows, the CTA rounds the earlier codes again under the new
// scale.  Scales are powers of two so that growing loses only what falls
// below the smallest code (a shift of an e4m3 exponent is exact), and
// appending a run row by row gives the scale that appending it at once does.
//
// Read.  The inverse on runs of positions: bf16 values code * 2^e (exact: a
// code has 4 significant bits).
//
// Bound: memory for long runs, the launch for a step.  A block to a CTA, since its
// scale needs all of its rows before the first code is written, and one CTA's registers
// hold them.  2,048 rows of 4 KV heads x 256 after 30,725 positions: append and read back
// together 7.4 us (21 MB: 3.1 us at the copy rate); one row to each of 32 requests 6.3 us;
// 32,768 x 4 rows read back 29 us, 6.9 TB/s with part of the writes left in L2.
#include "kv8.cuh"

namespace jfkv {

struct Kv8Args {
  uint8_t* pool;
  int64_t num_pages;
  int64_t page_bytes;
  int64_t codes_region;
  int64_t sb_region;
  int32_t P, log2P;
  int32_t Hkv;
  const int32_t* page_table;
  int32_t pt_stride;
  int32_t num_requests;
  const int32_t* start_pos;
  const int32_t* row_offsets;
  uint16_t* k;               // append: read; read back: written
  uint16_t* v;
  int64_t k_stride, v_stride;  // elements between rows
  int32_t n_rows;
  int32_t* err;
};

// Rows [r0, r1) of request b and its first position; false where they do not
// fit the row list, the request's page-table row or 31 bits.
__device__ __forceinline__ bool kv8_run(const Kv8Args& a, int b, int& r0, int& r1, int& pos0) {
  r0 = a.row_offsets[b];
  r1 = a.row_offsets[b + 1];
  pos0 = a.start_pos[b];
  return r0 >= 0 && r0 <= r1 && r1 <= a.n_rows && pos0 >= 0 &&
         (int64_t)pos0 + (r1 - r0) <= min((int64_t)a.pt_stride * a.P, (int64_t)0x7FFFFFFF);
}

template <int D>
__global__ void __launch_bounds__(256) kv8_append_kernel(const Kv8Args a) {
  constexpr int LPR = D / 8;               // lanes per row, 8 elements each
  constexpr int RPP = 256 / LPR;           // rows per pass
  constexpr int NP = KV8_BLOCK / RPP;      // passes over the block's 32 rows
  __shared__ uint32_t warp_max[8];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int head = blockIdx.y, kind = blockIdx.z;

  // the request and block this CTA takes: requests' block counts laid end to
  // end, 32 requests at a time (every warp works it out itself)
  int b = -1, r0 = 0, r1 = 0, pos0 = 0, blk = 0;
  for (int b0 = 0, base = 0; b0 < a.num_requests; b0 += 32) {
    const int bb = b0 + lane;
    int q0 = 0, q1 = 0, p0 = 0, n = 0;
    if (bb < a.num_requests) {
      if (kv8_run(a, bb, q0, q1, p0)) {
        if (q1 > q0) n = (p0 + (q1 - q0) - 1) / KV8_BLOCK - p0 / KV8_BLOCK + 1;
      } else if (blockIdx.x == 0 && head == 0 && kind == 0 && warp == 0) {
        flag_error(a.err, JF_DEV_ERR_POSITION);
      }
    }
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const int excl = base + incl - n;
    const unsigned m = __ballot_sync(0xffffffffu, n > 0 && (int)blockIdx.x >= excl &&
                                                      (int)blockIdx.x < excl + n);
    if (m && b < 0) {
      const int src = __ffs(m) - 1;
      b = b0 + src;
      r0 = __shfl_sync(0xffffffffu, q0, src);
      r1 = __shfl_sync(0xffffffffu, q1, src);
      pos0 = __shfl_sync(0xffffffffu, p0, src);
      blk = pos0 / KV8_BLOCK + (int)blockIdx.x - __shfl_sync(0xffffffffu, excl, src);
      if (blockIdx.x != 0) break;   // CTA 0 goes on to check every request
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (b < 0) return;

  const int block_pos = blk * KV8_BLOCK;
  const int first = max(pos0 - block_pos, 0);                          // new rows of the block:
  const int last = min(pos0 + (r1 - r0) - block_pos, KV8_BLOCK);       // [first, last)
  const int32_t page = a.page_table[(int64_t)b * a.pt_stride + (block_pos >> a.log2P)];
  if (page < 0 || page >= a.num_pages) {
    if (threadIdx.x == 0) flag_error(a.err, JF_DEV_ERR_PAGE_ID);
    return;
  }
  const int slot = block_pos & (a.P - 1);
  uint8_t* const rec = a.pool + (int64_t)page * a.page_bytes;
  uint8_t* const codes = rec + kind * a.codes_region + (int64_t)(head * a.P + slot) * D;
  float* const scale = reinterpret_cast<float*>(rec + 2 * a.codes_region + kind * a.sb_region) +
                       head * (a.P / KV8_BLOCK) + slot / KV8_BLOCK;

  const uint16_t* const src = kind ? a.v : a.k;
  const int64_t stride = kind ? a.v_stride : a.k_stride;
  const int li = threadIdx.x % LPR, rr = threadIdx.x / LPR;
  uint4 x[NP];
  uint32_t mx = 0;   // largest magnitude's bf16 bits (finite values only)
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int row = p * RPP + rr;
    x[p] = make_uint4(0u, 0u, 0u, 0u);
    if (row >= first && row < last)
      x[p] = *reinterpret_cast<const uint4*>(src + (int64_t)(r0 + block_pos + row - pos0) * stride +
                                             head * D + li * 8);
    const uint32_t w[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = w[i] & 0x7FFFu, hi = (w[i] >> 16) & 0x7FFFu;
      if (lo < 0x7F80u) mx = max(mx, lo);
      if (hi < 0x7F80u) mx = max(mx, hi);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  if (lane == 0) warp_max[warp] = mx;
  const int e_old = first > 0 ? exp8_of_scale(*scale) : KV8_EMIN;
  __syncthreads();   // every thread has read the old scale
#pragma unroll
  for (int i = 0; i < 8; ++i) mx = max(mx, warp_max[i]);
  const int e = max(e_old, exp8_of(__uint_as_float(mx << 16)));
  if (threadIdx.x == 0) *scale = two8(e);

  const float inv = two8(-e);
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int row = p * RPP + rr;
    if (row >= first && row < last) {
      uint2 c;
      c.x = e4m3x2(bf16lo_to_f32(x[p].x) * inv, bf16hi_to_f32(x[p].x) * inv) |
            (e4m3x2(bf16lo_to_f32(x[p].y) * inv, bf16hi_to_f32(x[p].y) * inv) << 16);
      c.y = e4m3x2(bf16lo_to_f32(x[p].z) * inv, bf16hi_to_f32(x[p].z) * inv) |
            (e4m3x2(bf16lo_to_f32(x[p].w) * inv, bf16hi_to_f32(x[p].w) * inv) << 16);
      *reinterpret_cast<uint2*>(codes + row * D + li * 8) = c;
    } else if (row < first && e > e_old) {   // the block grew: its earlier rows again
      uint2* const at = reinterpret_cast<uint2*>(codes + row * D + li * 8);
      uint2 c = *at;
      c.x = rescale_e4m3x4(c.x, e_old - e);
      c.y = rescale_e4m3x4(c.y, e_old - e);
      *at = c;
    }
  }
}

// Read back: a group of D/8 lanes takes the K and V vectors of KV8_RR rows and a
// KV head, 8 codes of each a lane, all rows' loads before their use.
constexpr int KV8_RR = 2;

template <int D>
__global__ void __launch_bounds__(256) kv8_read_kernel(const Kv8Args a) {
  constexpr int LPR = D / 8;
  constexpr int RPP = 256 / LPR;   // rows side by side
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int li = threadIdx.x % LPR;
  const int head = blockIdx.y;
  const int row0 = blockIdx.x * (RPP * KV8_RR) + threadIdx.x / LPR;
  uint2 c[KV8_RR][2];
  float s[KV8_RR][2];
  bool live[KV8_RR];
#pragma unroll
  for (int u = 0; u < KV8_RR; ++u) {
    const int row = row0 + u * RPP;
    live[u] = false;
    if (row >= a.n_rows) continue;
    // the request of this row: the last b with row_offsets[b] <= row
    int lo = 0, hi = a.num_requests - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.row_offsets[mid] <= row) lo = mid; else hi = mid - 1;
    }
    int r0, r1, pos0;
    const bool ok = kv8_run(a, lo, r0, r1, pos0);
    if (!ok || row < r0 || row >= r1) {
      if (!ok && li == 0) flag_error(a.err, JF_DEV_ERR_POSITION);
      continue;   // a row of no request is left as it is
    }
    const int pos = pos0 + (row - r0);
    const int32_t page = a.page_table[(int64_t)lo * a.pt_stride + (pos >> a.log2P)];
    if (page < 0 || page >= a.num_pages) {
      if (li == 0) flag_error(a.err, JF_DEV_ERR_PAGE_ID);
      continue;
    }
    live[u] = true;
    const int slot = pos & (a.P - 1);
    const uint8_t* const rec = a.pool + (int64_t)page * a.page_bytes;
    const uint8_t* const code = rec + (int64_t)(head * a.P + slot) * D + li * 8;
    const uint8_t* const scale =
        rec + 2 * a.codes_region + (head * (a.P / KV8_BLOCK) + slot / KV8_BLOCK) * 4;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      c[u][kind] = *reinterpret_cast<const uint2*>(code + kind * a.codes_region);
      s[u][kind] = *reinterpret_cast<const float*>(scale + kind * a.sb_region);
    }
  }
#pragma unroll
  for (int u = 0; u < KV8_RR; ++u) {
    if (!live[u]) continue;
    const int64_t row = row0 + u * RPP;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const float two = two8(exp8_of_scale(s[u][kind]));
      uint32_t h[4], o[4];
      f16x4_of_e4m3(c[u][kind].x, h[0], h[1]);
      f16x4_of_e4m3(c[u][kind].y, h[2], h[3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = f32x2_of_f16x2(h[i]);
        o[i] = pack_bf16x2_rn(f.x * two, f.y * two);
      }
      *reinterpret_cast<uint4*>((kind ? a.v : a.k) + row * (kind ? a.v_stride : a.k_stride) +
                                head * D + li * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

int launch_kv8_rows(const Geom& g, const jf_kv_pool& pool, const int32_t* page_table,
                    int32_t pt_stride, int32_t num_requests, const int32_t* start_pos,
                    const int32_t* row_offsets, void* k, int64_t k_stride, void* v,
                    int64_t v_stride, int32_t n_rows, int32_t* err, bool read,
                    cudaStream_t stream) {
  Kv8Args a;
  a.pool = static_cast<uint8_t*>(pool.base);
  a.num_pages = g.num_pages;
  a.page_bytes = g.page_bytes;
  a.codes_region = g.codes_region;
  a.sb_region = g.sb_region;
  a.P = g.P;
  a.log2P = __builtin_ctz((unsigned)g.P);
  a.Hkv = g.Hkv;
  a.page_table = page_table;
  a.pt_stride = pt_stride;
  a.num_requests = num_requests;
  a.start_pos = start_pos;
  a.row_offsets = row_offsets;
  a.k = static_cast<uint16_t*>(k);
  a.v = static_cast<uint16_t*>(v);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.n_rows = n_rows;
  a.err = err;
  // append: a request's r >= 1 rows touch at most (r - 1) / 32 + 2 blocks and
  // at most r; read: groups of D / 8 lanes, KV8_RR rows each
  const int64_t by_block = (int64_t)n_rows / KV8_BLOCK + 2 * (int64_t)num_requests;
  const int64_t per = KV8_RR * 256 / (g.D / 8);
  const int64_t blocks = read ? (n_rows + per - 1) / per
                              : (by_block < n_rows ? by_block : n_rows);
  if (blocks > 0x7FFFFFFF) return JF_ERR_UNSUPPORTED;
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, (unsigned)g.Hkv, read ? 1u : 2u);
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  cudaError_t e;
  if (read)
    e = g.D == 256 ? cudaLaunchKernelEx(&cfg, kv8_read_kernel<256>, a)
                   : cudaLaunchKernelEx(&cfg, kv8_read_kernel<128>, a);
  else
    e = g.D == 256 ? cudaLaunchKernelEx(&cfg, kv8_append_kernel<256>, a)
                   : cudaLaunchKernelEx(&cfg, kv8_append_kernel<128>, a);
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv
