// Rotary positions: pair j of a head at position p is turned by p f_j.
#include "operators.h"

namespace pbt {
namespace {

__global__ __launch_bounds__(256) void rotary_plan_kernel(RotaryFrequencies f, int n, double* __restrict__ table) {
  if ((int)threadIdx.x < n) table[threadIdx.x] = f.turns[threadIdx.x];
}

// cos and sin of p f: the product and the reduction to a quarter turn in double (at position 2^31 the product is good to 1e-7 of a turn, at a million to
// 1e-10), what is left, at most an eighth of a turn, in float
__device__ __forceinline__ float2 turn(double turns) {
  const double q = rint(4.0 * turns);
  const float r = (float)(4.0 * turns - q) * 0.5f;   // half turns, within +-1/4
  float s, c;
  sincospif(r, &s, &c);
  const int k = (int)(int64_t)q & 3;
  const float a = (k & 1) ? s : c, b = (k & 1) ? c : s;   // quarter turns: (c, s), (-s, c), (-c, -s), (s, -c)
  return make_float2(k == 1 || k == 2 ? -a : a, k >= 2 ? -b : b);
}

template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<bf16_t>(bf16_t v) { return bf2f(v); }
__device__ __forceinline__ void set(float* p, float v) { *p = v; }
__device__ __forceinline__ void set(bf16_t* p, float v) { *p = f2bf(v); }

__device__ __forceinline__ int64_t position(const RotaryArgs& a, int64_t row) {
  if (a.pos) return a.pos64 ? static_cast<const int64_t*>(a.pos)[row] : (int64_t)static_cast<const int32_t*>(a.pos)[row];
  return a.start + (a.period > 0 ? row % a.period : row);
}

// one workgroup a row, one thread a pair or an element of the part that is copied
template <class T, int LAYOUT>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  const int pairs = a.rot / 2, items = pairs + a.width - a.rot;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x)
  for (int k = threadIdx.x; k < items * a.heads; k += 256) {
    const double p = (double)position(a, row);
    int h = k / items, j = k % items, g = 0;
    while (h >= a.g[g].heads) h -= a.g[g++].heads;
    const T* src = static_cast<const T*>(a.g[g].d_src) + row * a.g[g].src_row + h * a.g[g].src_head;
    T* dst = static_cast<T*>(a.g[g].d_dst) + row * a.g[g].dst_row + h * a.g[g].dst_head;
    if (j >= pairs) {
      j += pairs;
      dst[j] = src[j];
      continue;
    }
    const float2 cs = turn(p * a.turns[j]);
    const float c = cs.x * a.gain, s = cs.y * a.gain * a.sign;
    const int e0 = LAYOUT == PBT_ROTARY_HALF ? j : 2 * j, e1 = LAYOUT == PBT_ROTARY_HALF ? j + pairs : 2 * j + 1;
    const float u = to_float(src[e0]), v = to_float(src[e1]);
    set(dst + e0, u * c - v * s);
    set(dst + e1, v * c + u * s);
  }
}

}  // namespace

hipError_t rotary_plan(const RotaryFrequencies& f, int n, double* table, hipStream_t s) {
  hipLaunchKernelGGL(rotary_plan_kernel, dim3(1), dim3(256), 0, s, f, n, table);
  return hipGetLastError();
}

hipError_t rotary_apply(const RotaryArgs& a, int layout, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20));
  if (dtype == PBT_DTYPE_BF16) {
    if (layout == PBT_ROTARY_HALF) hipLaunchKernelGGL((rotary_kernel<bf16_t, PBT_ROTARY_HALF>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<bf16_t, PBT_ROTARY_INTERLEAVED>), grid, dim3(256), 0, s, a);
  } else {
    if (layout == PBT_ROTARY_HALF) hipLaunchKernelGGL((rotary_kernel<float, PBT_ROTARY_HALF>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<float, PBT_ROTARY_INTERLEAVED>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace pbt
