// Block norms, backward, one pass over everything and a short sum of the parameters' gradients:
//   t = dout + N_pre^T(dz),  dx = alpha t,  v = beta a(gate) t,  dgate = beta a'(gate) u t,  dy = N_post^T(v)
//   N^T(w) = spread^-1 (w g - mean(w g) - hat mean(w g hat))   (RMS: without the first mean)
// u and out are formed again from y, x and the gate.  dz hat, dz, v hat, v (and u t for a gate vector) are summed over a slab's rows in registers; the
// slabs' sums go to `part`, and a second launch adds them in slab order.

#include "block_norm.h"

namespace pbt {
namespace {

constexpr int SUMS = 5;   // post gain, post bias, pre gain, pre bias, gate vector

template <class A, class R, int T, int J>
__global__ __launch_bounds__(block_threads(T)) void block_backward_kernel(BlockArgs a, int64_t rows_per_slab) {
  __shared__ float2 red[16];
  __shared__ float acc_lds[T <= 64 ? SUMS * T * J * 8 : 1];
  constexpr int GROUPS = block_threads(T) / T;
  const int i = blockIdx.y, l = threadIdx.x % T, group = threadIdx.x / T;
  const pbt_block_norm& k = a.n;
  const float inv_d = 1.f / (float)k.d;
  int ph = 0;
  int n[J];
  float g1[J][8], b1[J][8], g2[J][8], gv[J][8];
  float acc[SUMS][J][8];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = (l + T * j) * 8;
    n[j] = k.d - c;
    param8(a.p.post_gain, a.p.stride, i, c, n[j], 1.f, g1[j]);
    param8(a.p.post_bias, a.p.stride, i, c, n[j], 0.f, b1[j]);
    param8(a.p.pre_gain, a.p.stride, i, c, n[j], 1.f, g2[j]);
    if (k.gate == PBT_GATE_VECTOR) {
      float g[8];
      param8(a.p.gate, a.p.stride, i, c, n[j], 0.f, g);
      gate8<false>(k.gate_act, g, gv[j], nullptr);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) gv[j][e] = 1.f;
    }
#pragma unroll
    for (int q = 0; q < SUMS; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[q][j][e] = 0.f;
  }
  const int64_t r_end = min(k.rows, (int64_t)(blockIdx.x + 1) * rows_per_slab);
  for (int64_t r = blockIdx.x * rows_per_slab + group; r < r_end; r += GROUPS) {
    const int64_t row = i * k.rows + r;
    const float4 st = reinterpret_cast<const float4*>(a.stats)[row];
    float yh[J][8], xh[J][8], dz[J][8], t[J][8], f[J][8], df[J][8];
    Raw8<A> y[J], gate[J], dzr[J];
    Raw8<R> x[J], dout[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = (l + T * j) * 8;
      y[j].load(row_at<A>(a.y, row) + c, n[j]);
      x[j].load(row_at<R>(a.x, row) + c, n[j]);
      if (k.gate == PBT_GATE_ROWS) gate[j].load(row_at<A>(a.gate, row) + c, n[j]);
      if (a.dz.d) dzr[j].load(row_at<A>(a.dz, row) + c, n[j]);
      if (a.dout.d) dout[j].load(row_at<R>(a.dout, row) + c, n[j]);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float u[8];
      y[j].get(yh[j]);
      x[j].get(xh[j]);
      if (k.gate == PBT_GATE_ROWS) {
        float g[8];
        gate[j].get(g);
        gate8<true>(k.gate_act, g, f[j], df[j]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) { f[j][e] = gv[j][e]; df[j][e] = 1.f; }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        yh[j][e] = (yh[j][e] - st.x) * st.y;
        u[e] = k.post != PBT_NORM_NONE ? fmaf(yh[j][e], g1[j][e], b1[j][e]) : yh[j][e];
        const float o = fmaf(k.beta * f[j][e], u[e], k.alpha * xh[j][e]);
        xh[j][e] = (o - st.z) * st.w;
        df[j][e] *= u[e];
      }
      clear_past(yh[j], n[j]);
      clear_past(xh[j], n[j]);
      if (a.dz.d) {
        dzr[j].get(dz[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float w = dz[j][e] * g2[j][e];
          s1 += w;
          s2 = fmaf(w, xh[j][e], s2);
          t[j][e] = w;
          acc[2][j][e] = fmaf(dz[j][e], xh[j][e], acc[2][j][e]);
          acc[3][j][e] += dz[j][e];
        }
      }
    }
    if (a.dz.d) {
      const float2 m = row_sum2<T>(s1, s2, red, ph);
      s1 = k.pre == PBT_NORM_LAYER ? m.x * inv_d : 0.f;
      s2 = m.y * inv_d;
    }
    float q1 = 0.f, q2 = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = (l + T * j) * 8;
      float dx[8], dg[8], dv[8];
      if (a.dout.d) dout[j].get(dv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float s = a.dz.d ? st.w * (t[j][e] - s1 - xh[j][e] * s2) : 0.f;
        if (a.dout.d) s += dv[e];
        t[j][e] = s;
      }
      clear_past(t[j], n[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = t[j][e];
        dx[e] = k.alpha * s;
        dg[e] = k.beta * s * df[j][e];   // a'(g) u t
        acc[4][j][e] += dg[e];
        const float v = k.beta * f[j][e] * s;
        acc[0][j][e] = fmaf(v, yh[j][e], acc[0][j][e]);
        acc[1][j][e] += v;
        const float w = v * g1[j][e];
        q1 += w;
        q2 = fmaf(w, yh[j][e], q2);
        t[j][e] = k.post != PBT_NORM_NONE ? w : v;
      }
      put8(row_at<R>(a.dx, row) + c, dx, n[j]);
      if (k.gate == PBT_GATE_ROWS) put8(row_at<A>(a.dgate, row) + c, dg, n[j]);
    }
    if (k.post != PBT_NORM_NONE) {
      const float2 m = row_sum2<T>(q1, q2, red, ph);
      q1 = k.post == PBT_NORM_LAYER ? m.x * inv_d : 0.f;
      q2 = m.y * inv_d;
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = (l + T * j) * 8;
      if (k.post != PBT_NORM_NONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[j][e] = st.y * (t[j][e] - q1 - yh[j][e] * q2);
      }
      put8(row_at<A>(a.dy, row) + c, t[j], n[j]);
    }
  }
  // the gate vector's slope is the same for all rows
  if (k.gate == PBT_GATE_VECTOR) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float g[8], f[8], df[8];
      param8(a.p.gate, a.p.stride, i, (l + T * j) * 8, n[j], 0.f, g);
      gate8<true>(k.gate_act, g, f, df);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[4][j][e] *= df[e];
    }
  }
  float* const* grads = &a.g.post_gain;
  float* part = a.part + ((int64_t)i * gridDim.x + blockIdx.x) * SUMS * k.d;
  if (T <= 64) {
    // groups of a workgroup take turns
    for (int turn = 0; turn < GROUPS; ++turn) {
      if (group == turn) {
#pragma unroll
        for (int q = 0; q < SUMS; ++q)
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float* p = acc_lds + (q * J + j) * T * 8 + l * 8 + e;
              *p = turn == 0 ? acc[q][j][e] : *p + acc[q][j][e];
            }
      }
      __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < SUMS; ++q)
      if (grads[q])
        for (int c = threadIdx.x; c < k.d; c += block_threads(T)) part[q * k.d + c] = acc_lds[q * J * T * 8 + c];
  } else {
#pragma unroll
    for (int q = 0; q < SUMS; ++q)
      if (grads[q]) {
#pragma unroll
        for (int j = 0; j < J; ++j) put8(part + q * k.d + (l + T * j) * 8, acc[q][j], n[j]);
      }
  }
}

// adds the slabs' sums in slab order: a workgroup covers 64 columns of one parameter of one member, its four wavefronts a quarter of the slabs each
__global__ __launch_bounds__(256) void block_param_kernel(const float* __restrict__ part, int slabs, int d, pbt_block_params g) {
  __shared__ float red[4][64];
  float* const out = (&g.post_gain)[blockIdx.y];
  if (!out) return;
  const int i = blockIdx.z, cl = threadIdx.x & 63, grp = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + cl;
  const int per = (slabs + 3) / 4, k_end = min(slabs, (grp + 1) * per);
  float acc = 0.f;
  if (c < d)
    for (int k = grp * per; k < k_end; ++k) acc += part[((int64_t)(i * (int64_t)slabs + k) * SUMS + blockIdx.y) * d + c];
  red[grp][cl] = acc;
  __syncthreads();
  if (grp == 0 && c < d) out[i * g.stride + c] = ((red[0][cl] + red[1][cl]) + red[2][cl]) + red[3][cl];
}

int64_t slabs_of(const pbt_block_norm& n) {
  const BlockShape b = block_shape(n.d);
  const int groups = block_threads(b.T) / b.T;
  const int64_t most = 1024 / n.P + 1;
  const int64_t s = (n.rows + groups - 1) / groups;
  return s < most ? s : most;
}

template <class A, class R, int T, int J>
void launch(const BlockArgs& a, int64_t slabs, hipStream_t s) {
  const int64_t rows_per_slab = (a.n.rows + slabs - 1) / slabs;
  hipLaunchKernelGGL((block_backward_kernel<A, R, T, J>), dim3((unsigned)slabs, a.n.P), dim3(block_threads(T)), 0, s, a, rows_per_slab);
}
template <class A, class R>
void by_width(const BlockArgs& a, int64_t slabs, hipStream_t s) {
  const BlockShape b = block_shape(a.n.d);
  if (b.T == 16) launch<A, R, 16, 1>(a, slabs, s);
  else if (b.T == 64) b.J == 1 ? launch<A, R, 64, 1>(a, slabs, s) : launch<A, R, 64, 2>(a, slabs, s);
  else if (b.T == 256) b.J == 1 ? launch<A, R, 256, 1>(a, slabs, s) : launch<A, R, 256, 2>(a, slabs, s);
  else launch<A, R, 512, 2>(a, slabs, s);
}

}  // namespace

size_t block_norm_work_bytes(const pbt_block_norm& n) { return (size_t)n.P * slabs_of(n) * SUMS * n.d * sizeof(float); }

hipError_t block_norm_backward(const BlockArgs& a, hipStream_t s) {
  const int64_t slabs = slabs_of(a.n);
  if (slabs > 0) {
    const bool act16 = a.n.dtype == PBT_DTYPE_BF16, res16 = a.n.res_dtype == PBT_DTYPE_BF16;
    if (act16) res16 ? by_width<bf16_t, bf16_t>(a, slabs, s) : by_width<bf16_t, float>(a, slabs, s);
    else res16 ? by_width<float, bf16_t>(a, slabs, s) : by_width<float, float>(a, slabs, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const pbt_block_params& g = a.g;
  if (g.post_gain || g.post_bias || g.pre_gain || g.pre_bias || g.gate)
    hipLaunchKernelGGL(block_param_kernel, dim3((a.n.d + 63) / 64, SUMS, a.n.P), dim3(256), 0, s, a.part, (int)slabs, a.n.d, g);
  return hipGetLastError();
}

}  // namespace pbt
