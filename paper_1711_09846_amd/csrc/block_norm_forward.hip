// Block norms, forward: u = N_post(y), out = alpha x + beta a(gate) u, z = N_pre(out) in one pass over y, x and the gate.

#include "block_norm.h"

namespace pbt {
namespace {

template <class A, class R, int T, int J>
__global__ __launch_bounds__(block_threads(T)) void block_forward_kernel(BlockArgs a, int64_t rows_per_slab) {
  __shared__ float2 red[16];
  constexpr int GROUPS = block_threads(T) / T;   // rows at a time
  const int i = blockIdx.y, l = threadIdx.x % T, group = threadIdx.x / T;
  const pbt_block_norm& k = a.n;
  const float d = (float)k.d;
  int ph = 0;
  int n[J];
  float g1[J][8], b1[J][8], g2[J][8], b2[J][8], gv[J][8];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = (l + T * j) * 8;
    n[j] = k.d - c;
    param8(a.p.post_gain, a.p.stride, i, c, n[j], 1.f, g1[j]);
    param8(a.p.post_bias, a.p.stride, i, c, n[j], 0.f, b1[j]);
    param8(a.p.pre_gain, a.p.stride, i, c, n[j], 1.f, g2[j]);
    param8(a.p.pre_bias, a.p.stride, i, c, n[j], 0.f, b2[j]);
    if (k.gate == PBT_GATE_VECTOR) {
      float g[8];
      param8(a.p.gate, a.p.stride, i, c, n[j], 0.f, g);
      gate8<false>(k.gate_act, g, gv[j], nullptr);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) gv[j][e] = 1.f;
    }
  }
  const int64_t r_end = min(k.rows, (int64_t)(blockIdx.x + 1) * rows_per_slab);
  for (int64_t r = blockIdx.x * rows_per_slab + group; r < r_end; r += GROUPS) {
    const int64_t row = i * k.rows + r;
    float u[J][8], o[J][8];
    Raw8<A> gate[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = (l + T * j) * 8;
      Raw8<A> y;
      Raw8<R> x;
      y.load(row_at<A>(a.y, row) + c, n[j]);
      x.load(row_at<R>(a.x, row) + c, n[j]);
      if (k.gate == PBT_GATE_ROWS) gate[j].load(row_at<A>(a.gate, row) + c, n[j]);
      y.get(u[j]);
      x.get(o[j]);
    }
    float2 s1 = make_float2(0.f, 1.f), s2 = make_float2(0.f, 1.f);
    if (k.post != PBT_NORM_NONE) s1 = row_stats<T, J>(u, n, k.post, d, k.eps, red, ph);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = (l + T * j) * 8;
      float f[8];
      if (k.gate == PBT_GATE_ROWS) {
        float g[8];
        gate[j].get(g);
        gate8<false>(k.gate_act, g, f, nullptr);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = gv[j][e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (k.post != PBT_NORM_NONE) u[j][e] = fmaf(u[j][e] * s1.y, g1[j][e], b1[j][e]);
        o[j][e] = fmaf(k.beta * f[e], u[j][e], k.alpha * o[j][e]);
      }
      put8(row_at<R>(a.out, row) + c, o[j], n[j]);
    }
    if (k.pre != PBT_NORM_NONE) {
      s2 = row_stats<T, J>(o, n, k.pre, d, k.eps, red, ph);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = (l + T * j) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[j][e] = fmaf(o[j][e] * s2.y, g2[j][e], b2[j][e]);
        put8(row_at<A>(a.z, row) + c, o[j], n[j]);
      }
    }
    if (a.stats && l == 0) reinterpret_cast<float4*>(a.stats)[row] = make_float4(s1.x, s1.y, s2.x, s2.y);
  }
}

template <class A, class R, int T, int J>
hipError_t launch(const BlockArgs& a, hipStream_t s) {
  constexpr int GROUPS = block_threads(T) / T;
  const int64_t most = 2048 / a.n.P + 1;   // slabs of a member: a few workgroups for every compute unit, all members together
  int64_t slabs = (a.n.rows + GROUPS - 1) / GROUPS;
  if (slabs > most) slabs = most;
  const int64_t rows_per_slab = (a.n.rows + slabs - 1) / slabs;
  hipLaunchKernelGGL((block_forward_kernel<A, R, T, J>), dim3((unsigned)slabs, a.n.P), dim3(block_threads(T)), 0, s, a, rows_per_slab);
  return hipGetLastError();
}
template <class A, class R>
hipError_t by_width(const BlockArgs& a, hipStream_t s) {
  const BlockShape b = block_shape(a.n.d);
  if (b.T == 16) return launch<A, R, 16, 1>(a, s);
  if (b.T == 64) return b.J == 1 ? launch<A, R, 64, 1>(a, s) : launch<A, R, 64, 2>(a, s);
  if (b.T == 256) return b.J == 1 ? launch<A, R, 256, 1>(a, s) : launch<A, R, 256, 2>(a, s);
  return launch<A, R, 512, 2>(a, s);
}

}  // namespace

hipError_t block_norm_forward(const BlockArgs& a, hipStream_t s) {
  const bool act16 = a.n.dtype == PBT_DTYPE_BF16, res16 = a.n.res_dtype == PBT_DTYPE_BF16;
  if (act16) return res16 ? by_width<bf16_t, bf16_t>(a, s) : by_width<bf16_t, float>(a, s);
  return res16 ? by_width<float, bf16_t>(a, s) : by_width<float, float>(a, s);
}

}  // namespace pbt
