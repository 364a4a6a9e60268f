// Append to and read back from the latent cache.
//
// Append and read copy rows of R + 64 bf16 values between the caller's latent and
// key parts and the pages: one 16-byte piece a thread, its row's request found by
// bisection, so that runs of any lengths need no plan.  Bound: a launch and dependent
// loads: the bisection's, log2 of the requests (5 at 32, 12 at 4,096), its request's
// start, the page, the row.  Both calls for 32 rows of 576 channels
// take 4.4 us, for 2,048 rows (9.4 MB moved in all, 1.4 us at copy rate) 4.2 us.
#include "latent.cuh"

namespace jfkv {

struct LatentRows {
  uint16_t* pool;
  int64_t num_pages;
  int32_t P, log2P;
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

}  // namespace jfkv
