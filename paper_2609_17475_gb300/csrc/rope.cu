// Rotary positions with several axes (time, height, width) on query and key
// rows, and their gradient (the inverse rotation).
//
// Pair i of a head's first R channels is a point (x, y) turned by the angle
// pos[axis_i, t] * f_i:  (x cos - y sin, x sin + y cos); channels past R pass
// through.  The angle depends on the token alone, so a CTA works out the R/2
// cosines and sines of its token once in shared memory and turns every query
// and key head with them, 16 bytes of a row per thread and step.
//
// The angle is kept as a fraction of a turn in 64-bit fixed point: the host
// rounds f_i / (2 pi) to a multiple of 2^-64 and pos * that, modulo 2^64, is
// exact integer arithmetic, so a far position loses nothing (an fp32 product
// is off by 0.01 rad at position 262,144) and no range reduction is needed.
//
// Bound by memory: each element is read and written once.
#include "common.cuh"

namespace jfkv {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_PAIRS = 128;

struct RopeSide {
  const uint8_t* in;
  uint8_t* out;
  int64_t in_token, in_head;     // strides in elements
  int64_t out_token, out_head;
  int32_t heads;
};

struct RopeArgs {
  const int32_t* pos;
  int64_t pos_stride;            // elements between the axes' rows
  int32_t n_tokens;
  int32_t D;                     // channels per head
  int32_t R;                     // rotated channels
  int32_t adjacent;              // pairs (2i, 2i+1) instead of (i, i + R/2)
  int32_t inverse;
  RopeSide side[2];              // queries, keys
  uint64_t turn[ROPE_MAX_PAIRS]; // turns per position, in units of 2^-64
  uint8_t axis[ROPE_MAX_PAIRS];
};

template <typename T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Elem<__half> {
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
};
template <> struct Elem<float> {
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};

template <typename T>
union Vec16 {
  uint4 w;
  T e[16 / sizeof(T)];
  __device__ Vec16() : w(make_uint4(0u, 0u, 0u, 0u)) {}
};

template <typename T>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float2 cs[ROPE_MAX_PAIRS];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int64_t t = blockIdx.x;
  const int half = a.R / 2;
  for (int i = threadIdx.x; i < half; i += ROPE_THREADS) {
    const int32_t p = a.pos[a.axis[i] * a.pos_stride + t];
    const uint64_t turns = (uint64_t)(int64_t)p * a.turn[i];
    // the nearest signed fraction of a turn, in half turns
    const float x = (float)(int32_t)(turns >> 32) * 4.656612873077393e-10f;   // 2^-31
    float s, c;
    sincospif(x, &s, &c);
    cs[i] = make_float2(c, a.inverse ? -s : s);
  }
  __syncthreads();
  // steps of a head: half pairing turns two vectors at once; then the
  // channels that pass through
  const int turn_steps = a.adjacent ? a.R / V : half / V;
  const int steps = turn_steps + (a.D - a.R) / V;
  const int heads = a.side[0].heads + a.side[1].heads;
  for (int u = threadIdx.x; u < heads * steps; u += ROPE_THREADS) {
    const int h = u / steps, k = u % steps;
    const bool key = h >= a.side[0].heads;
    const RopeSide& sd = a.side[key];
    const int hh = key ? h - a.side[0].heads : h;
    const T* in = reinterpret_cast<const T*>(sd.in) + t * sd.in_token + hh * sd.in_head;
    T* out = reinterpret_cast<T*>(sd.out) + t * sd.out_token + hh * sd.out_head;
    if (k >= turn_steps) {
      const int d = a.R + (k - turn_steps) * V;
      if (in != out)
        *reinterpret_cast<uint4*>(out + d) = *reinterpret_cast<const uint4*>(in + d);
    } else if (a.adjacent) {
      Vec16<T> x, y;
      x.w = *reinterpret_cast<const uint4*>(in + k * V);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float2 w = cs[k * (V / 2) + i];
        const float p = Elem<T>::get(x.e[2 * i]), q = Elem<T>::get(x.e[2 * i + 1]);
        y.e[2 * i] = Elem<T>::put(p * w.x - q * w.y);
        y.e[2 * i + 1] = Elem<T>::put(p * w.y + q * w.x);
      }
      *reinterpret_cast<uint4*>(out + k * V) = y.w;
    } else {
      Vec16<T> x0, x1, y0, y1;
      x0.w = *reinterpret_cast<const uint4*>(in + k * V);
      x1.w = *reinterpret_cast<const uint4*>(in + half + k * V);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 w = cs[k * V + i];
        const float p = Elem<T>::get(x0.e[i]), q = Elem<T>::get(x1.e[i]);
        y0.e[i] = Elem<T>::put(p * w.x - q * w.y);
        y1.e[i] = Elem<T>::put(p * w.y + q * w.x);
      }
      *reinterpret_cast<uint4*>(out + k * V) = y0.w;
      *reinterpret_cast<uint4*>(out + half + k * V) = y1.w;
    }
  }
}

// f / (2 pi) modulo 1, rounded to a multiple of 2^-64
static uint64_t turns_per_position(float f) {
  const double t = (double)f * 0.15915494309189533577;   // 1 / (2 pi)
  double frac = t - (double)(int64_t)t;                  // |t| < 2^62 (checked by the caller)
  if (frac < 0.0) frac += 1.0;
  if (frac >= 1.0) return 0;
  // two 32-bit pieces: 2^64 itself does not fit
  const double hi = frac * 4294967296.0;
  const uint64_t h = (uint64_t)hi;
  const uint64_t l = (uint64_t)((hi - (double)h) * 4294967296.0);
  return (h << 32) | l;
}

int launch_rope(const jf_rope& rope, const int32_t* positions, int64_t pos_stride,
                int32_t n_tokens, int32_t head_dim, const jf_rope_rows& q, const jf_rope_rows& k,
                int32_t dtype, int32_t inverse, cudaStream_t stream) {
  RopeArgs a;
  a.pos = positions;
  a.pos_stride = pos_stride;
  a.n_tokens = n_tokens;
  a.D = head_dim;
  a.R = rope.rotary_dim;
  a.adjacent = rope.pairing == JF_ROPE_PAIR_ADJACENT;
  a.inverse = inverse != 0;
  const jf_rope_rows* rows[2] = {&q, &k};
  for (int s = 0; s < 2; ++s) {
    RopeSide& d = a.side[s];
    d.in = static_cast<const uint8_t*>(rows[s]->in);
    d.out = static_cast<uint8_t*>(rows[s]->out);
    d.in_token = rows[s]->in_token_stride;
    d.in_head = rows[s]->in_head_stride;
    d.out_token = rows[s]->out_token_stride;
    d.out_head = rows[s]->out_head_stride;
    d.heads = rows[s]->num_heads;
  }
  for (int i = 0; i < ROPE_MAX_PAIRS; ++i) {
    const bool on = i < a.R / 2;
    a.turn[i] = on ? turns_per_position(rope.inv_freq[i]) : 0;
    a.axis[i] = on ? (uint8_t)rope.axis[i] : 0;
  }
  cudaLaunchAttribute pdl[1];
  pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_tokens);
  cfg.blockDim = dim3(ROPE_THREADS);
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  cudaError_t e;
  switch (dtype) {
    case JF_DTYPE_BF16: e = cudaLaunchKernelEx(&cfg, rope_kernel<__nv_bfloat16>, a); break;
    case JF_DTYPE_F16: e = cudaLaunchKernelEx(&cfg, rope_kernel<__half>, a); break;
    default: e = cudaLaunchKernelEx(&cfg, rope_kernel<float>, a); break;
  }
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv
