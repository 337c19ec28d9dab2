// What both passes of the block norms share (block_norm_forward.hip, block_norm_backward.hip): how a row lies over threads, sums over a row, the gate.
//
// A row of d elements lies in the registers of T threads, eight consecutive elements in each of J places: thread l has columns (l + T j) 8 .. + 7.  T = 16
// (four rows a wavefront) for up to 128 columns, a wavefront for up to 1024, workgroups of 256 and 512 threads for up to 4096 and 8192, so
// that a row is read once whatever is summed over it.  A workgroup takes a slab of a member's rows; a thread keeps the same
// columns for all of them, so parameters are read once a slab and their gradients add up in registers.
#pragma once
#include "operators.h"

namespace pbt {

struct BlockShape { int T, J; };
inline BlockShape block_shape(int d) {
  if (d <= 128) return {16, 1};
  if (d <= 512) return {64, 1};
  if (d <= 1024) return {64, 2};
  if (d <= 2048) return {256, 1};
  if (d <= 4096) return {256, 2};
  return {512, 2};
}
constexpr int block_threads(int T) { return T < 256 ? 256 : T; }

// sums of two values over the T threads of a row, to all of them; red: 2 x 8 float2 of LDS, ph: which half is used (rows wider than a wavefront: a
// barrier a call; the halves alternate, so that a wavefront can be one sum ahead of another but not two)
template <int T>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* red, int& ph) {
  const auto dpp = [](float v, auto ctrl) { return v + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
  if (T == 16) {
    a = dpp(a, std::integral_constant<int, 0x128>()); b = dpp(b, std::integral_constant<int, 0x128>());
    a = dpp(a, std::integral_constant<int, 0x124>()); b = dpp(b, std::integral_constant<int, 0x124>());
    a = dpp(a, std::integral_constant<int, 0x4e>()); b = dpp(b, std::integral_constant<int, 0x4e>());
    a = dpp(a, std::integral_constant<int, 0xb1>()); b = dpp(b, std::integral_constant<int, 0xb1>());
    return make_float2(a, b);
  }
  a = wave_sum(a);
  b = wave_sum(b);
  if (T == 64) return make_float2(a, b);
  float2* r = red + 8 * ph;
  ph ^= 1;
  if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  float2 t = r[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) { t.x += r[w].x; t.y += r[w].y; }
  return t;
}

// the gate's factor a(g), and a'(g) (SLOPE)
template <bool SLOPE>
__device__ __forceinline__ void gate8(int act, const float* g, float* f, float* df) {
  switch (act) {
    case PBT_ACT_TANH:
#pragma unroll
      for (int e = 0; e < 8; ++e) { f[e] = tanhf(g[e]); if (SLOPE) df[e] = 1.f - f[e] * f[e]; }
      break;
    case PBT_ACT_SIGMOID:
#pragma unroll
      for (int e = 0; e < 8; ++e) { f[e] = 1.f / (1.f + expf(-g[e])); if (SLOPE) df[e] = f[e] * (1.f - f[e]); }
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

// eight parameters of a member from column c, or `otherwise` where there are none; zero past the row's end
__device__ __forceinline__ void param8(const float* p, int64_t stride, int member, int c, int n, float otherwise, float* v) {
  if (p) {
    Raw8<float> r;
    r.load(p + member * stride + c, n);
    r.get(v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = otherwise;
    clear_past(v, n);
  }
}

template <class T> __device__ __forceinline__ T* row_at(const pbt_rows& m, int64_t row) { return static_cast<T*>(m.d) + row * m.pitch; }

// statistics of a row in registers: mean (LAYER; else 0) and 1 / sqrt(variance or mean square + eps); the values become (v - mean).  The variance is summed
// over the differences, a second sum: no cancellation.  (Divisions: the mean of a row of equal
// values is that value, which a reciprocal's rounding would not give.)
template <int T, int J>
__device__ __forceinline__ float2 row_stats(float (*v)[8], const int* n, int kind, float d, float eps, float2* red, int& ph) {
  float mean = 0.f;
  if (kind == PBT_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[j][e];
    mean = row_sum2<T>(s, 0.f, red, ph).x / d;
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] -= mean;
      clear_past(v[j], n[j]);
    }
  }
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) q = fmaf(v[j][e], v[j][e], q);
  return make_float2(mean, rsqrtf(row_sum2<T>(q, 0.f, red, ph).x / d + eps));
}

}  // namespace pbt
