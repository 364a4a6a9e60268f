// Rotary positions with several axes (time, height, width) on query and key
// rows, and their gradient (the inverse rotation).
//
// Pair i of a head's first R channels is a point (x, y) turned by the angle
// pos[axis_i, t] * f_i:  (x cos - y sin, x sin + y cos); channels past R pass
// through.  The angle depends on the token alone, so a CTA works out the R/2
// cosines and sines of its tokens once in shared memory and turns every query
// and key head with them, 16 bytes of a row (two pieces with half pairing) per
// thread and step.
//
// The angle is kept as a fraction of a turn in 64-bit fixed point: the host
// rounds f_i / (2 pi) to a multiple of 2^-64 and pos * that, modulo 2^64, is
// exact integer arithmetic, so the product is off by at most 2^-34 of a turn at
// any position (an fp32 product by 0.01 rad at position 262,144) and no range
// reduction is needed.  Its upper 32 bits become an fp32 in half turns, which
// rounds to 2^-26 of a turn.
//
// Bound by memory: each element is read and written once.  2,048 tokens of 28 heads x
// 256 (bf16, all channels turned) 12.6 us, 4.7 TB/s, of which about 4 us are the launch
// and the first loads (32 tokens: 4.1 us); the gradient of 16,391 tokens of 20 heads x
// 128 (fp16) 33.3 us, 5.0 TB/s.  One CTA a token (two, where that fills the SMs anyway)
// keeps the cosines beside the heads that use them: 18 KB of rows a CTA, many CTAs an SM.
#include <cstring>

#include "common.cuh"

namespace jfkv {

int sm_count();

constexpr int ROPE_THREADS = 128;
constexpr int ROPE_MAX_PAIRS = 128;
constexpr int ROPE_MAX_TPB = 2;     // tokens per CTA

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
  int32_t tpb;                   // tokens per CTA
  int32_t D;                     // channels per head
  int32_t R;                     // rotated channels
  int32_t adjacent;              // pairs (2i, 2i+1) instead of (i, i + R/2)
  int32_t inverse;
  RopeSide side[2];              // queries, keys
  uint64_t turn[ROPE_MAX_PAIRS]; // turns per position, in units of 2^-64
  uint8_t axis[ROPE_MAX_PAIRS];
};

// 16 bytes of elements <-> fp32, two elements an instruction where there is one
template <typename T> struct Pack;
template <> struct Pack<__nv_bfloat16> {
  static __device__ __forceinline__ void get(uint32_t w, float* x) {
    x[0] = bf16lo_to_f32(w);
    x[1] = bf16hi_to_f32(w);
  }
  static __device__ __forceinline__ uint32_t put(const float* x) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(x[1]), "f"(x[0]));
    return r;
  }
};
template <> struct Pack<__half> {
  static __device__ __forceinline__ void get(uint32_t w, float* x) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    x[0] = f.x;
    x[1] = f.y;
  }
  static __device__ __forceinline__ uint32_t put(const float* x) { return pack_f16x2(x[0], x[1]); }
};
template <> struct Pack<float> {
  static __device__ __forceinline__ void get(uint32_t w, float* x) { x[0] = __uint_as_float(w); }
  static __device__ __forceinline__ uint32_t put(const float* x) { return __float_as_uint(x[0]); }
};
template <typename T>
__device__ __forceinline__ void unpack16(const uint4& v, float (&x)[16 / sizeof(T)]) {
  constexpr int E = 4 / sizeof(T);   // elements of a word
  Pack<T>::get(v.x, x);
  Pack<T>::get(v.y, x + E);
  Pack<T>::get(v.z, x + 2 * E);
  Pack<T>::get(v.w, x + 3 * E);
}
template <typename T>
__device__ __forceinline__ uint4 pack16(const float (&x)[16 / sizeof(T)]) {
  constexpr int E = 4 / sizeof(T);
  return make_uint4(Pack<T>::put(x), Pack<T>::put(x + E), Pack<T>::put(x + 2 * E),
                    Pack<T>::put(x + 3 * E));
}

// `tpb` tokens a CTA.  Threads 0 .. per * steps - 1 work: thread u has place
// u % steps of every per-th of the CTA's (token, head) pairs, the next pair's
// loads issued before the current one is turned.
template <typename T, bool ADJ>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int V = 16 / sizeof(T);
  constexpr int NC = ADJ ? V / 2 : V;      // pairs of a place
  __shared__ __align__(16) float2 cs[ROPE_MAX_TPB * ROPE_MAX_PAIRS];
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int half = a.R / 2;
  const int64_t t0 = (int64_t)blockIdx.x * a.tpb;
  const int nt = (int)min((int64_t)a.tpb, a.n_tokens - t0);
  // places of a head: those turned, then the channels that pass through
  const int turned = ADJ ? a.R / V : half / V;
  const int steps = turned + (a.D - a.R) / V;
  const int per = ROPE_THREADS / steps;    // pairs side by side (D <= 512: at least one)
  const int h0 = threadIdx.x / steps, k = threadIdx.x - h0 * steps;
  const int hq = a.side[0].heads, heads = hq + a.side[1].heads;
  const bool turn = k < turned;
  const int d = turn ? k * V : a.R + (k - turned) * V;
  const bool second = !ADJ && turn;
  // (token j, head h) -> its input and output places
  auto place = [&](int j, int h, const T*& in, T*& out) {
    const RopeSide& sd = a.side[h >= hq];
    const int hh = h >= hq ? h - hq : h;
    in = reinterpret_cast<const T*>(sd.in) + (t0 + j) * sd.in_token + hh * sd.in_head + d;
    out = reinterpret_cast<T*>(sd.out) + (t0 + j) * sd.out_token + hh * sd.out_head + d;
  };
  int j = 0, h = h0;
  auto settle = [&]() {
    while (h >= heads) {
      h -= heads;
      ++j;
    }
  };
  settle();
  bool live = h0 < per && j < nt;
  const T* in = nullptr;
  T* out = nullptr;
  uint4 v0 = make_uint4(0u, 0u, 0u, 0u), v1 = v0;
  if (live) {
    place(j, h, in, out);
    v0 = *reinterpret_cast<const uint4*>(in);
    if (second) v1 = *reinterpret_cast<const uint4*>(in + half);
  }
  for (int u = threadIdx.x; u < nt * half; u += ROPE_THREADS) {
    const int jj = u / half, i = u - jj * half;
    const int32_t p = a.pos[a.axis[i] * a.pos_stride + t0 + jj];
    const uint64_t turns = (uint64_t)(int64_t)p * a.turn[i];
    // the nearest signed fraction of a turn, in half turns
    const float x = (float)(int32_t)(turns >> 32) * 4.656612873077393e-10f;   // 2^-31
    float s, c;
    sincospif(x, &s, &c);
    // in twos, those of neighbouring places adjoining, so that the loads below meet no
    // bank twice (a place's pairs in a row: 13.9 us for the 2,048 tokens, not 12.6; kept
    // in registers across a token's heads: 12.7, and the gradient 36.2, not 33.3)
    cs[jj * half + 2 * (i % NC / 2 * turned + i / NC) + (i & 1)] =
        make_float2(c, a.inverse ? -s : s);
  }
  __syncthreads();
  while (live) {
    const uint4 x0 = v0, x1 = v1;
    T* const to = out;
    const bool same = in == out;
    const int jc = j;
    h += per;
    settle();
    live = j < nt;
    if (live) {
      place(j, h, in, out);
      v0 = *reinterpret_cast<const uint4*>(in);
      if (second) v1 = *reinterpret_cast<const uint4*>(in + half);
    }
    if (turn) {
      const float4* const w = reinterpret_cast<const float4*>(cs + jc * half) + k;
      float p0[V], p1[V], y0[V], y1[V];
      unpack16<T>(x0, p0);
      if (!ADJ) unpack16<T>(x1, p1);
#pragma unroll
      for (int i = 0; i < NC; i += 2) {
        const float4 f = w[i / 2 * turned];   // cosine and sine of pairs i and i + 1
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float c = e ? f.z : f.x, s = e ? f.w : f.y;
          const float p = ADJ ? p0[2 * (i + e)] : p0[i + e];
          const float q = ADJ ? p0[2 * (i + e) + 1] : p1[i + e];
          const float r0 = p * c - q * s, r1 = p * s + q * c;
          if (ADJ) {
            y0[2 * (i + e)] = r0;
            y0[2 * (i + e) + 1] = r1;
          } else {
            y0[i + e] = r0;
            y1[i + e] = r1;
          }
        }
      }
      *reinterpret_cast<uint4*>(to) = pack16<T>(y0);
      if (!ADJ) *reinterpret_cast<uint4*>(to + half) = pack16<T>(y1);
    } else if (!same) {
      *reinterpret_cast<uint4*>(to) = x0;
    }
  }
}

// f / (2 pi) modulo 1, rounded to a multiple of 2^-64.  f = m 2^x with a whole m below 2^24, and
// 1 / (2 pi) to 128 bits, so that the product is good to 2^-104 of a turn times 2^x, x <= 8.
static uint64_t turns_per_position(float f) {
  typedef unsigned __int128 u128;
  const u128 inv = ((u128)0x28BE60DB9391054AULL << 64) | 0x7F09D5F47D4D3770ULL;   // 2^128 / (2 pi)
  uint32_t b;
  memcpy(&b, &f, 4);
  const int e = (int)(b >> 23) & 0xFF, x = (e ? e : 1) - 150;
  const u128 m = (b & 0x7FFFFFu) | (e ? 0x800000u : 0u);
  // m inv 2^(x - 64) in units of 2^-64, modulo 2^64: m inv in two parts of 64 bits and what is above
  const u128 lo = m * (uint64_t)inv, hi = m * (uint64_t)(inv >> 64) + (lo >> 64);   // hi below 2^88
  const int shift = 64 - x;                                   // 56 (|f| below 2^32) and up
  uint64_t turns = 0;
  if (shift <= 64) {
    const u128 low = (hi << 64) | (uint64_t)lo;               // the product's low 128 bits
    turns = (uint64_t)(low >> shift) + ((uint64_t)(low >> (shift - 1)) & 1u);
  } else if (shift - 64 <= 88) {
    turns = (uint64_t)(hi >> (shift - 64)) + ((uint64_t)(hi >> (shift - 65)) & 1u);
  }
  return f < 0.f ? 0 - turns : turns;
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
  // One token a CTA, or two in long runs, where the start of a CTA weighs more
  // (16,391 tokens of 20 heads x 128: 34.0 us with one, 33.3 with two; 2,048
  // tokens of 28 x 256: 12.6 us with one, 15.1 with two).
  a.tpb = n_tokens >= 16 * sm_count() ? 2 : 1;
  cfg.gridDim = dim3((unsigned)((n_tokens + a.tpb - 1) / a.tpb));
  cfg.blockDim = dim3(ROPE_THREADS);
  cfg.stream = stream;
  cfg.attrs = pdl;
  cfg.numAttrs = 1;
  cudaError_t e;
  const bool adj = a.adjacent != 0;
  switch (dtype) {
    case JF_DTYPE_BF16:
      e = adj ? cudaLaunchKernelEx(&cfg, rope_kernel<__nv_bfloat16, true>, a)
              : cudaLaunchKernelEx(&cfg, rope_kernel<__nv_bfloat16, false>, a);
      break;
    case JF_DTYPE_F16:
      e = adj ? cudaLaunchKernelEx(&cfg, rope_kernel<__half, true>, a)
              : cudaLaunchKernelEx(&cfg, rope_kernel<__half, false>, a);
      break;
    default:
      e = adj ? cudaLaunchKernelEx(&cfg, rope_kernel<float, true>, a)
              : cudaLaunchKernelEx(&cfg, rope_kernel<float, false>, a);
      break;
  }
  return e == cudaSuccess ? JF_OK : JF_ERR_CUDA;
}

}  // namespace jfkv
