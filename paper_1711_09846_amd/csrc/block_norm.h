// What both passes of the block norms share (block_norm_forward.hip, block_norm_backward.hip): how a row lies over threads, sums over a row, the gate.
//
// A thread has eight consecutive elements of a row in registers, so that a row is read once whatever is summed over it.  A team of T threads has a row: 8, 16 or 32 of a
// wavefront's (rows of up to 64, 128, 256 elements), a wavefront (up to 512), or as many wavefronts as the row needs, one workgroup (WIDE, up to 16
// wavefronts).  A workgroup takes a slab of a member's rows; a thread keeps the same columns for all of them, so parameters are read once a slab and
// their gradients add up in registers.  The next row is requested as soon as this one's values have been taken over: loads are single instructions without a
// branch around their results, which the compiler would wait at (with such branches 8191 rows of 5001 took 129 us forward, 94 without, 88 now).
#pragma once
#include "operators.h"

namespace pbt {

// over T = 8, 16 or 32 adjacent lanes: quads change places, half rows are mirrored (quads are equal by then), rows of 16 are mirrored, two rows are swapped
template <int T>
__device__ __forceinline__ float lanes_sum(float v) {
  const auto f = [](float x, auto ctrl) { return x + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
  v = f(v, std::integral_constant<int, 0xb1>());             // quad_perm [1, 0, 3, 2]
  v = f(v, std::integral_constant<int, 0x4e>());             // quad_perm [2, 3, 0, 1]
  v = f(v, std::integral_constant<int, 0x141>());            // row_half_mirror
  if (T >= 16) v = f(v, std::integral_constant<int, 0x140>());   // row_mirror
  if (T >= 32) {
    const auto g = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(g[0]) + __uint_as_float(g[1]);
  }
  return v;
}

// Sums of two values over a team, to all its threads.  WIDE teams: a barrier a sum; wavefronts leave their sums in one of two halves of LDS by turns, so that
// one wavefront can be a sum ahead of another but not two.
template <int T> struct TeamSum {
  __device__ __forceinline__ TeamSum(float2*) {}
  __device__ __forceinline__ float2 operator()(float a, float b) {
    return T < 64 ? make_float2(lanes_sum<T>(a), lanes_sum<T>(b)) : make_float2(wave_sum(a), wave_sum(b));
  }
};
template <> struct TeamSum<WIDE> {
  float2* red;   // [2][16]
  int half = 0;
  __device__ __forceinline__ TeamSum(float2* lds) : red(lds) {
    if (threadIdx.x < 32) red[threadIdx.x] = make_float2(0.f, 0.f);
    __syncthreads();
  }
  __device__ __forceinline__ float2 operator()(float a, float b) {
    a = wave_sum(a);
    b = wave_sum(b);
    float2* r = red + 16 * half;
    half ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    const float2 v = r[threadIdx.x & 15];
    return make_float2(lanes_sum<16>(v.x), lanes_sum<16>(v.y));
  }
};

// The gate's factor a(g), and a'(g) (SLOPE).  Slopes keep their relative precision where the gate is nearly 1, as differences from 1 would not:
// 1 - tanh(g)^2 = e^(-2|g|) (1 + |tanh g|)^2, by 4 |g| + 8 half steps (the exponent's rounding), and 1 - sigmoid(g) = e^(-g) sigmoid(g).
template <bool SLOPE>
__device__ __forceinline__ void gate8(int act, const float* g, float* f, float* df) {
  switch (act) {
    case PBT_ACT_TANH:
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[e] = tanhf(g[e]);
        if (SLOPE) {
          const float q = 1.f + fabsf(f[e]);
          df[e] = __builtin_amdgcn_exp2f(-2.88539008f * fabsf(g[e])) * q * q;
        }
      }
      break;
    case PBT_ACT_SIGMOID:
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = expf(-g[e]);
        f[e] = 1.f / (1.f + t);
        if (SLOPE) df[e] = f[e] > 0.f ? t * f[e] * f[e] : f[e];   // (0 where t is infinite)
      }
      break;
    case PBT_ACT_SILU:
#pragma unroll
      for (int e = 0; e < 8; ++e) { const float s = 1.f / (1.f + expf(-g[e])); f[e] = g[e] * s; if (SLOPE) df[e] = s * (1.f + g[e] * (1.f - s)); }
      break;
    default:
#pragma unroll
      for (int e = 0; e < 8; ++e) { f[e] = g[e]; if (SLOPE) df[e] = 1.f; }
  }
}

// elements past the row's end (n of the eight exist) to zero
__device__ __forceinline__ void clear_past(float* v, int n) {
  if (n < 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= n) v[e] = 0.f;
  }
}

// How a wavefront reads a row's eight elements a lane.  The lane at the row's end reads the eight that end there, its neighbours' among them: those must be
// of the same wavefront, whose loads come before its stores (another one may have written its part already where an output lies over the input).
// ALONE (block_ends_alone): widths whose last wavefront has fewer than eight elements in all, which are read one by one.
template <bool ALONE> struct RowReader {
  bool alone;   // this is that wavefront
  int n;
  __device__ __forceinline__ RowReader(int left) : alone(ALONE && __builtin_amdgcn_readfirstlane(left) < 8), n(left) {}
  template <class T> __device__ __forceinline__ void load(Raw8<T>& r, const T* p) const {
    if (ALONE && alone) r.load(p, n);
    else r.load_end(p, n);
  }
  template <class T> __device__ __forceinline__ void get(const Raw8<T>& r, float* v) const {
    if (ALONE && alone) r.get(v);
    else get_end(r, v, n);
  }
};

// Eight parameters of a member from column c, or `otherwise` where there are none; zero past the row's end.  All of a kernel's are requested before the first
// is looked at.
template <class Reader>
__device__ __forceinline__ void load_param(const Reader& reader, Raw8<float>& r, const float* p, int64_t stride, int member, int c) {
  if (p) reader.load(r, p + member * stride + c);
}
template <class Reader>
__device__ __forceinline__ void get_param(const Reader& reader, const Raw8<float>& r, const float* p, float otherwise, float* v) {
  if (p) {
    reader.get(r, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = otherwise;
    clear_past(v, reader.n);
  }
}

template <class T> __device__ __forceinline__ T* row_at(const pbt_rows& m, int64_t row) { return static_cast<T*>(m.d) + row * m.pitch; }

// Statistics of a row: mean (LAYER; else 0) and 1 / sqrt(variance or mean square + eps); the values become v - mean.  The variance is summed over the
// differences, a second sum: no cancellation.  (Divisions: the mean of a row of equal values is that value, which a reciprocal's rounding would not
// give.)
template <class Sum>
__device__ __forceinline__ float2 row_stats(float* v, int n, int kind, float d, float eps, Sum& sum) {
  float mean = 0.f;
  if (kind == PBT_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e];
    mean = sum(s, 0.f).x / d;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] -= mean;
    clear_past(v, n);
  }
  float q = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) q = fmaf(v[e], v[e], q);
  return make_float2(mean, rsqrtf(sum(q, 0.f).x / d + eps));
}

}  // namespace pbt
