// Append to and read back from the latent cache, and attention over it one query
// row at a time.
//
// Append and read copy rows of R + 64 bf16 values between the caller's latent and
// key parts and the pages: one 16-byte piece a thread.  Bound: the launch for a
// step, memory for long runs.
#include "latent.cuh"

namespace jfkv {

struct LatentRows {
  uint16_t* pool;
  int64_t num_pages;
  int32_t P, log2P, R;
  const int32_t* page_table;
  int32_t pt_stride, num_requests;
  const int32_t* start_pos;
  const int32_t* row_offsets;
  uint16_t* latent;
  uint16_t* k_rot;
  int64_t latent_stride, rot_stride;
  int32_t n_rows;
  int32_t* err;
};

constexpr int LR_THREADS = 288;   // 4 rows of R = 512 (72 pieces each), 7 of 256 (40 each)

template <int R, bool READ>
__global__ void __launch_bounds__(LR_THREADS) latent_rows_kernel(const LatentRows a) {
  constexpr int PIECES = (R + LAT_ROT) / 8;
  constexpr int ROWS = LR_THREADS / PIECES;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if (blockIdx.x == 0)   // every request's run is checked, those without rows too
    for (int b = threadIdx.x; b < a.num_requests; b += LR_THREADS) {
      const int r0 = a.row_offsets[b], r1 = a.row_offsets[b + 1], pos0 = a.start_pos[b];
      if (!(r0 >= 0 && r0 <= r1 && r1 <= a.n_rows && pos0 >= 0 &&
            (int64_t)pos0 + (r1 - r0) <= min((int64_t)a.pt_stride * a.P, (int64_t)0x7FFFFFFF)))
        flag_error(a.err, JF_DEV_ERR_POSITION);
    }
  const int piece = threadIdx.x % PIECES;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / PIECES;
  if (threadIdx.x >= ROWS * PIECES || row >= a.n_rows) return;
  // the request of this row: the last b with row_offsets[b] <= row
  int lo = 0, hi = a.num_requests - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.row_offsets[mid] <= row) lo = mid; else hi = mid - 1;
  }
  const int r0 = a.row_offsets[lo], r1 = a.row_offsets[lo + 1], pos0 = a.start_pos[lo];
  if (r0 < 0 || row < r0 || row >= r1 || r1 > a.n_rows || pos0 < 0 ||
      (int64_t)pos0 + (r1 - r0) > min((int64_t)a.pt_stride * a.P, (int64_t)0x7FFFFFFF))
    return;   // a row of no request, or of one that is flagged
  const int pos = pos0 + (int)(row - r0);
  const int32_t page = a.page_table[(int64_t)lo * a.pt_stride + (pos >> a.log2P)];
  if (page < 0 || page >= a.num_pages) {
    if (piece == 0) flag_error(a.err, JF_DEV_ERR_PAGE_ID);
    return;
  }
  uint4* const at = reinterpret_cast<uint4*>(
      a.pool + ((int64_t)page * a.P + (pos & (a.P - 1))) * (R + LAT_ROT) + piece * 8);
  uint4* const own = reinterpret_cast<uint4*>(
      piece < R / 8 ? a.latent + row * a.latent_stride + piece * 8
                    : a.k_rot + row * a.rot_stride + (piece - R / 8) * 8);
  if (READ)
    *own = *at;
  else
    *at = *own;
}

int launch_latent_rows(const LatentPool& pool, const int32_t* page_table, int32_t pt_stride,
                       int32_t num_requests, const int32_t* start_pos, const int32_t* row_offsets,
                       void* latent, int64_t latent_stride, void* k_rot, int64_t rot_stride,
                       int32_t n_rows, int32_t* err, bool read, cudaStream_t stream) {
  LatentRows a;
  a.pool = const_cast<uint16_t*>(pool.base);
  a.num_pages = pool.num_pages;
  a.P = pool.P;
  a.log2P = pool.log2P;
  a.R = pool.R;
  a.page_table = page_table;
  a.pt_stride = pt_stride;
  a.num_requests = num_requests;
  a.start_pos = start_pos;
  a.row_offsets = row_offsets;
  a.latent = static_cast<uint16_t*>(latent);
  a.k_rot = static_cast<uint16_t*>(k_rot);
  a.latent_stride = latent_stride;
  a.rot_stride = rot_stride;
  a.n_rows = n_rows;
  a.err = err;
  const int64_t per = LR_THREADS / (pool.row / 8);
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((n_rows + per - 1) / per));
  cfg.blockDim = dim3(LR_THREADS);
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  cudaError_t e;
  if (read)
    e = pool.R == 512 ? cudaLaunchKernelEx(&cfg, latent_rows_kernel<512, true>, a)
                      : cudaLaunchKernelEx(&cfg, latent_rows_kernel<256, true>, a);
  else
    e = pool.R == 512 ? cudaLaunchKernelEx(&cfg, latent_rows_kernel<512, false>, a)
                      : cudaLaunchKernelEx(&cfg, latent_rows_kernel<256, false>, a);
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

// ---------------------------------------------------------------------------
// One query row a CTA: 8 warps take every eighth position, a lane (R + 64) / 32
// channels, with a running maximum and sum each; the warps' results are joined at
// the end.
// ---------------------------------------------------------------------------
constexpr int LS_WARPS = 8;

template <int R>
struct RowSmem {
  float q[R + LAT_ROT];
  float o[LS_WARPS][R];
  float m[LS_WARPS], l[LS_WARPS];
};

template <int R>
struct RowState {
  float m = -INFINITY, l = 0.f, o[R / 32];
};

template <int R>
__device__ void row_run(const LatentPool& p, const int32_t* pt, int n, RowSmem<R>& s,
                        RowState<R>& st, int32_t* status) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int t = warp; t < n; t += LS_WARPS) {
    const int32_t page = pt[t >> p.log2P];
    if (page < 0 || page >= p.num_pages) {
      if (lane == 0) flag_error(status, JF_DEV_ERR_PAGE_ID);
      continue;
    }
    const uint16_t* const row = p.base + ((int64_t)page * p.P + (t & (p.P - 1))) * (R + LAT_ROT);
    float x = 0.f, c[R / 32];
#pragma unroll
    for (int i = 0; i < (R + LAT_ROT) / 64; ++i) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(row + i * 64 + lane * 2);
      const float lo = bf16lo_to_f32(w), hi = bf16hi_to_f32(w);
      x = fmaf(lo, s.q[i * 64 + lane * 2], x);
      x = fmaf(hi, s.q[i * 64 + lane * 2 + 1], x);
      if (i < R / 64) {
        c[2 * i] = lo;
        c[2 * i + 1] = hi;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    const float m = x > st.m ? x : st.m;
    const float f = m == -INFINITY ? 1.f : exp2f(st.m - m);
    const float w = x == -INFINITY ? 0.f : exp2f(x - m);   // NaN stays
    st.m = m;
    st.l = fmaf(st.l, f, w);
#pragma unroll
    for (int i = 0; i < R / 32; ++i) st.o[i] = fmaf(st.o[i], f, w * c[i]);
  }
}

// the warps' states joined: s.o[0][channel] = the normalized output
template <int R>
__device__ void row_join(RowSmem<R>& s, RowState<R>& st) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) {
    s.m[warp] = st.m;
    s.l[warp] = st.l;
  }
#pragma unroll
  for (int i = 0; i < R / 64; ++i) {
    s.o[warp][i * 64 + lane * 2] = st.o[2 * i];
    s.o[warp][i * 64 + lane * 2 + 1] = st.o[2 * i + 1];
  }
  __syncthreads();
  float m = -INFINITY, l = 0.f;
  for (int w = 0; w < LS_WARPS; ++w) m = fmaxf(m, s.m[w]);
  for (int w = 0; w < LS_WARPS; ++w) l += s.l[w] * (s.m[w] == -INFINITY ? 1.f : exp2f(s.m[w] - m));
  for (int c = threadIdx.x; c < R; c += blockDim.x) {
    float o = 0.f;
    for (int w = 0; w < LS_WARPS; ++w)
      o += s.o[w][c] * (s.m[w] == -INFINITY ? 1.f : exp2f(s.m[w] - m));
    s.o[0][c] = l == 0.f ? 0.f : o / l;
  }
  __syncthreads();
}

template <int R>
__global__ void __launch_bounds__(32 * LS_WARPS)
latent_prefill_rows_kernel(const __grid_constant__ LatentPrefill a) {
  __shared__ RowSmem<R> s;
  const int h = blockIdx.y, i = blockIdx.x;
  const uint16_t* const q = a.q + ((int64_t)i * a.H + h) * (LAT_HEAD + LAT_ROT);
  const uint16_t* const wk = a.w_k + (int64_t)h * LAT_HEAD * R;
  const uint16_t* const wv = a.w_v + (int64_t)h * LAT_HEAD * R;
  for (int c = threadIdx.x; c < R; c += blockDim.x) {
    float x = 0.f;
    for (int k = 0; k < LAT_HEAD; ++k)
      x = fmaf(__uint_as_float((uint32_t)q[k] << 16), __uint_as_float((uint32_t)wk[k * R + c] << 16), x);
    s.q[c] = x * a.scale_log2;
  }
  for (int c = threadIdx.x; c < LAT_ROT; c += blockDim.x)
    s.q[R + c] = __uint_as_float((uint32_t)q[LAT_HEAD + c] << 16) * a.scale_log2;
  __syncthreads();
  RowState<R> st;
  for (int c = 0; c < R / 32; ++c) st.o[c] = 0.f;
  row_run<R>(a.pool, a.pt, a.causal ? a.q_start + i + 1 : a.q_start + a.C, s, st, a.status);
  row_join<R>(s, st);
  for (int v = threadIdx.x; v < LAT_HEAD; v += blockDim.x) {
    float x = 0.f;
    for (int c = 0; c < R; ++c) x = fmaf(s.o[0][c], __uint_as_float((uint32_t)wv[v * R + c] << 16), x);
    a.out[((int64_t)i * a.H + h) * LAT_HEAD + v] = (uint16_t)pack_bf16x2(x, 0.f);
  }
}

size_t latent_prefill_workspace_bytes(int64_t, int64_t, int64_t, int64_t) { return 256; }

int launch_latent_prefill(const LatentPrefill& a, void*, cudaStream_t stream) {
  const dim3 grid((unsigned)a.C, (unsigned)a.H);
  if (a.pool.R == 512)
    latent_prefill_rows_kernel<512><<<grid, 32 * LS_WARPS, 0, stream>>>(a);
  else
    latent_prefill_rows_kernel<256><<<grid, 32 * LS_WARPS, 0, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv
