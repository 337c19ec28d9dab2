// Block norms, backward, one pass over everything and a short sum of the parameters' gradients:
//   t = dout + N_pre^T(dz),  dx = alpha t,  v = beta a(gate) t,  dgate = beta a'(gate) u t,  dy = N_post^T(v)
//   N^T(w) = spread^-1 (w g - mean(w g) - hat mean(w g hat))   (RMS: without the first mean)
// u and out are formed again from y, x and the gate.  dz hat, dz, v hat, v (and dgate for a gate vector) are summed over a slab's rows in registers; the
// slabs' sums go to `part`, and a second launch adds them in slab order.  The parameters wait in LDS: a compute unit gets some eight bytes a cycle from memory
// and 128 from LDS, registers are what limits how many rows are on their way.
// Bound by memory: 16 x 4096 rows of 512 with a gate a row and the stream in fp32, 738 MB: 150 us (4.9 TB/s); 16384 rows of 2048: 131 (4.6); 8191 rows of 5001:
// 118 (4.2).  33.5 million elements in rows of 64 take 127 us, of 32 154, of 16 243, of 8 384.  The second launch: 4 to 10 us.
#include <type_traits>

#include "block_norm.h"
#include "gemm_common.h"

namespace pbt {
namespace {

constexpr int SUMS = 5;     // post gain, post bias, pre gain, pre bias, gate vector
constexpr int PARAMS = 4;   // post gain, post bias, pre gain, the gate's factor

__device__ __forceinline__ void from_lds(const float4* lds, int stride, int which, int l, float* v) {
  const float4 a = lds[(2 * which) * stride + l], b = lds[(2 * which + 1) * stride + l];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void to_lds(float4* lds, int stride, int which, int l, const float* v) {
  lds[(2 * which) * stride + l] = make_float4(v[0], v[1], v[2], v[3]);
  lds[(2 * which + 1) * stride + l] = make_float4(v[4], v[5], v[6], v[7]);
}

// ALL: every parameter's gradient; else those of the two gains only
template <class A, class R, int T, int MOST, bool ALL, bool ALONE>
__global__ __launch_bounds__(MOST) void block_backward_kernel(BlockArgs a, int64_t rows_per_slab) {
  extern __shared__ float4 lds[];   // [PARAMS][2][threads of a team], then the team's sums
  constexpr int ROWS = T == WIDE ? 1 : 256 / T;
  const int team = T == WIDE ? (int)blockDim.x : T;
  __shared__ float2 red[32];
  TeamSum<T> sum(red);
  const int i = blockIdx.y, l = T == WIDE ? threadIdx.x : threadIdx.x % T, group = T == WIDE ? 0 : threadIdx.x / T;
  const pbt_block_norm& k = a.n;
  const float inv_d = 1.f / (float)k.d;
  const int c = l * 8, n = k.d - c;
  const RowReader<ALONE> reader(n);
  const bool rows_gate = k.gate == PBT_GATE_ROWS, has_dz = a.dz.d != nullptr, has_dout = a.dout.d != nullptr;
  const int64_t r_end = min(k.rows, (int64_t)(blockIdx.x + 1) * rows_per_slab);
  Raw8<A> y, gate, dzr;
  Raw8<R> x, dout;
  float4 st_next;
  auto fetch = [&](int64_t r) {
    const int64_t row = i * k.rows + r;
    st_next = reinterpret_cast<const float4*>(a.stats)[row];
    reader.load(y, row_at<A>(a.y, row) + c);
    reader.load(x, row_at<R>(a.x, row) + c);
    if (rows_gate) reader.load(gate, row_at<A>(a.gate, row) + c);
    if (has_dz) reader.load(dzr, row_at<A>(a.dz, row) + c);
  };
  auto fetch_dout = [&](int64_t r) {
    if (has_dout) reader.load(dout, row_at<R>(a.dout, i * k.rows + r) + c);
  };
  int64_t r = blockIdx.x * rows_per_slab + group;
  if (r < r_end) {
    fetch(r);
    fetch_dout(r);
  }
  if (group == 0) {
    Raw8<float> raw[4];
    const float* const at[4] = {a.p.post_gain, a.p.post_bias, a.p.pre_gain, k.gate == PBT_GATE_VECTOR ? a.p.gate : nullptr};
    float p[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) load_param(reader, raw[q], at[q], a.p.stride, i, c);
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      get_param(reader, raw[q], at[q], q == 1 ? 0.f : 1.f, p);
      to_lds(lds, team, q, l, p);
    }
    if (k.gate == PBT_GATE_VECTOR) {
      float g[8];
      get_param(reader, raw[3], at[3], 0.f, g);
      gate8<false>(k.gate_act, g, p, nullptr);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = 1.f;
    }
    to_lds(lds, team, 3, l, p);
  }
  __syncthreads();
  float acc[SUMS][8];
#pragma unroll
  for (int q = 0; q < SUMS; ++q)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[q][e] = 0.f;
  for (; r < r_end; r += ROWS) {
    const int64_t row = i * k.rows + r;
    const float4 st = st_next;
    float yh[8], xh[8], t[8], f[8], df[8], p[8], q[8];
    reader.get(y, yh);
    reader.get(x, xh);
    if (rows_gate) {
      reader.get(gate, p);
      gate8<true>(k.gate_act, p, f, df);
    } else {
      from_lds(lds, team, 3, l, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) df[e] = 1.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) yh[e] = (yh[e] - st.x) * st.y;
    float u[8];
    if (k.post != PBT_NORM_NONE) {
      from_lds(lds, team, 0, l, p);
      from_lds(lds, team, 1, l, q);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = fmaf(yh[e], p[e], q[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = yh[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      xh[e] = (fmaf(k.beta * f[e], u[e], k.alpha * xh[e]) - st.z) * st.w;
      df[e] *= u[e];
    }
    clear_past(yh, n);
    clear_past(xh, n);
    float s1 = 0.f, s2 = 0.f;
    if (has_dz) {
      float dz[8];
      reader.get(dzr, dz);
      from_lds(lds, team, 2, l, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t[e] = dz[e] * p[e];
        s1 += t[e];
        s2 = fmaf(t[e], xh[e], s2);
        acc[2][e] = fmaf(dz[e], xh[e], acc[2][e]);
        if (ALL) acc[3][e] += dz[e];
      }
    }
    if (r + ROWS < r_end) fetch(r + ROWS);   // (on its way while this row is reduced)
    if (has_dz) {
      const float2 m = sum(s1, s2);
      s1 = k.pre == PBT_NORM_LAYER ? m.x * inv_d : 0.f;
      s2 = m.y * inv_d;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = st.w * (t[e] - s1 - xh[e] * s2);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = 0.f;
    }
    if (has_dout) {
      float dv[8];
      reader.get(dout, dv);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] += dv[e];
    }
    if (r + ROWS < r_end) fetch_dout(r + ROWS);
    clear_past(t, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      xh[e] = k.alpha * t[e];             // dx
      df[e] = k.beta * t[e] * df[e];      // dgate
      t[e] = k.beta * f[e] * t[e];        // v
      if (ALL) acc[4][e] += df[e];
      acc[0][e] = fmaf(t[e], yh[e], acc[0][e]);
      if (ALL) acc[1][e] += t[e];
    }
    put8(row_at<R>(a.dx, row) + c, xh, n);
    if (rows_gate) put8(row_at<A>(a.dgate, row) + c, df, n);
    if (k.post != PBT_NORM_NONE) {
      from_lds(lds, team, 0, l, p);
      float q1 = 0.f, q2 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t[e] *= p[e];
        q1 += t[e];
        q2 = fmaf(t[e], yh[e], q2);
      }
      const float2 m = sum(q1, q2);
      q1 = k.post == PBT_NORM_LAYER ? m.x * inv_d : 0.f;
      q2 = m.y * inv_d;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = st.y * (t[e] - q1 - yh[e] * q2);
    }
    put8(row_at<A>(a.dy, row) + c, t, n);
  }
  // the gate vector's slope is the same for all rows
  if (k.gate == PBT_GATE_VECTOR) {
    float g[8], f[8], df[8];
    Raw8<float> raw;
    load_param(reader, raw, a.p.gate, a.p.stride, i, c);
    get_param(reader, raw, a.p.gate, 0.f, g);
    gate8<true>(k.gate_act, g, f, df);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[4][e] *= df[e];
  }
  float* const* grads = &a.g.post_gain;
  float* part = a.part + ((int64_t)i * gridDim.x + blockIdx.x) * SUMS * k.d;
  if (T != WIDE) {
    // the teams of a workgroup add theirs up: those of a wavefront across its lanes, then the wavefronts in turn
#pragma unroll
    for (int by = T; by < 64; by *= 2)
#pragma unroll
      for (int q = 0; q < SUMS; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[q][e] += __shfl_xor(acc[q][e], by);
    const int wave = threadIdx.x >> 6;
    __syncthreads();   // (the parameters in LDS have been used)
    for (int turn = 0; turn < 4; ++turn) {
      if (wave == turn && (threadIdx.x & 63) < T) {
#pragma unroll
        for (int q = 0; q < SUMS; ++q) {
          float v[8];
          if (turn > 0) {
            from_lds(lds, team, q, l, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[q][e] = v[e] + acc[q][e];
          }
          if (turn < 3) to_lds(lds, team, q, l, acc[q]);
          else if (grads[q]) put8(part + q * k.d + c, acc[q], n);
        }
      }
      __syncthreads();
    }
  } else {
#pragma unroll
    for (int q = 0; q < SUMS; ++q)
      if (grads[q]) put8(part + q * k.d + c, acc[q], n);
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
  if (c < d) {
    const float* __restrict__ p = part + ((int64_t)i * slabs * SUMS + blockIdx.y) * d + c;
    for (int k = grp * per; k < k_end; k += 8) {   // (eight loads on their way)
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = k + q < k_end ? p[(int64_t)(k + q) * SUMS * d] : 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) acc += v[q];
    }
  }
  red[grp][cl] = acc;
  __syncthreads();
  if (grp == 0 && c < d) out[i * g.stride + c] = ((red[0][cl] + red[1][cl]) + red[2][cl]) + red[3][cl];
}

int64_t slabs_of(const pbt_block_norm& n) { return (n.rows + block_backward_slab(n) - 1) / block_backward_slab(n); }

// more than 64 KB of LDS need a permission, once on every device (wide teams have 72 to 128 KB, whose compute unit has no room for a second of them anyway)
template <class A, class R, int MOST, bool ALL, bool ALONE>
hipError_t launch_wide(const BlockArgs& a, int64_t per_slab, dim3 grid, dim3 block, size_t lds, hipStream_t s) {
  if (lds > 64 * 1024) {
    const hipError_t e = allow_lds<&block_backward_kernel<A, R, WIDE, MOST, ALL, ALONE>>(128 * 1024);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((block_backward_kernel<A, R, WIDE, MOST, ALL, ALONE>), grid, block, lds, s, a, per_slab);
  return hipGetLastError();
}
template <class A, class R>
hipError_t launch(const BlockArgs& a, int64_t slabs, hipStream_t s) {
  const BlockTeam t = block_team(a.n.d);
  const int64_t per_slab = block_backward_slab(a.n);
  const dim3 grid((unsigned)slabs, a.n.P), block(t.threads);
  const size_t lds = (size_t)(t.T == WIDE ? PARAMS : SUMS) * 2 * (t.T == WIDE ? t.threads : t.T) * sizeof(float4);
  // (Widths that end alone have one instance, for every size of a workgroup and all sums, whose registers spill.  16352 rows of 513: 138 us, 16130 of 520 60;
  // 8184 of 1025 114, 8128 of 1032 48; 4094 of 2049 90, 4080 of 2056 45.)
  if (block_ends_alone(a.n.d)) {
    if (t.T == WIDE) return launch_wide<A, R, 1024, true, true>(a, per_slab, grid, block, lds, s);
    hipLaunchKernelGGL((block_backward_kernel<A, R, 8, 256, true, true>), grid, block, lds, s, a, per_slab);
  } else if (t.T == 8) hipLaunchKernelGGL((block_backward_kernel<A, R, 8, 256, true, false>), grid, block, lds, s, a, per_slab);
  else if (t.T == 32) hipLaunchKernelGGL((block_backward_kernel<A, R, 32, 256, true, false>), grid, block, lds, s, a, per_slab);
  else if (t.T == 16) hipLaunchKernelGGL((block_backward_kernel<A, R, 16, 256, true, false>), grid, block, lds, s, a, per_slab);
  else if (t.T == 64) hipLaunchKernelGGL((block_backward_kernel<A, R, 64, 256, true, false>), grid, block, lds, s, a, per_slab);
  else if (t.threads <= 512) return launch_wide<A, R, 512, true, false>(a, per_slab, grid, block, lds, s);
  else if (t.threads <= 768) return launch_wide<A, R, 768, true, false>(a, per_slab, grid, block, lds, s);
  // (1024 threads have 128 registers each: with all five sums some go to memory.  2 x 2048 rows of 7000: 155 us with two sums, 282 with five; up to 768
  // threads the number makes no difference)
  else if (a.g.post_bias || a.g.pre_bias || a.g.gate) return launch_wide<A, R, 1024, true, false>(a, per_slab, grid, block, lds, s);
  else return launch_wide<A, R, 1024, false, false>(a, per_slab, grid, block, lds, s);
  return hipGetLastError();
}

}  // namespace

size_t block_norm_work_bytes(const pbt_block_norm& n) { return (size_t)n.P * slabs_of(n) * SUMS * n.d * sizeof(float); }

hipError_t block_norm_backward(const BlockArgs& a, hipStream_t s) {
  const int64_t slabs = slabs_of(a.n);
  if (slabs > 0) {
    const bool act16 = a.n.dtype == PBT_DTYPE_BF16, res16 = a.n.res_dtype == PBT_DTYPE_BF16;
    const hipError_t e = act16 ? (res16 ? launch<bf16_t, bf16_t>(a, slabs, s) : launch<bf16_t, float>(a, slabs, s))
                               : (res16 ? launch<float, bf16_t>(a, slabs, s) : launch<float, float>(a, slabs, s));
    if (e != hipSuccess) return e;
  }
  const pbt_block_params& g = a.g;
  if (g.post_gain || g.post_bias || g.pre_gain || g.pre_bias || g.gate)
    hipLaunchKernelGGL(block_param_kernel, dim3((a.n.d + 63) / 64, SUMS, a.n.P), dim3(256), 0, s, a.part, (int)slabs, a.n.d, g);
  return hipGetLastError();
}

}  // namespace pbt
