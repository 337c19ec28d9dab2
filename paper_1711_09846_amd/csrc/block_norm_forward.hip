// Block norms, forward: u = N_post(y), out = alpha x + beta a(gate) u, z = N_pre(out) in one pass over y, x and the gate.
// Bound by memory: 16 x 4096 rows of 512 bf16 with a gate vector, 268 MB: 53 to 59 us; with a gate a row and the stream in fp32, 470 MB: 88 (5.3 TB/s); 16384 rows of
// 2048: 84 (4.8).  Rows of thousands of elements cost what their addresses do: 8191 rows of 5120, which begin at whole lines of memory, take 70 us (4.8 TB/s), of 5000 81,
// of 5001 88 (3.7).  Narrow rows leave lanes idle, a team has at least eight: 33.5 million elements in rows of 64 take 45 us, of 32 66, of 16 116, of 8 207.  4 rows of
// 2048: 3.4 us.
#include <type_traits>

#include "block_norm.h"

namespace pbt {
namespace {

template <class A, class R, int T, int MOST, bool ALONE>
__global__ __launch_bounds__(MOST) void block_forward_kernel(BlockArgs a, int64_t rows_per_slab) {
  __shared__ float2 red[32];
  TeamSum<T> sum(red);
  constexpr int ROWS = T == WIDE ? 1 : 256 / T;   // rows at a time
  const int i = blockIdx.y, l = T == WIDE ? threadIdx.x : threadIdx.x % T, group = T == WIDE ? 0 : threadIdx.x / T;
  const pbt_block_norm& k = a.n;
  const float d = (float)k.d;
  const int c = l * 8, n = k.d - c;   // the thread's columns, how many of them there are (n <= 0: none)
  const RowReader<ALONE> reader(n);
  const bool rows_gate = k.gate == PBT_GATE_ROWS;
  const int64_t r_end = min(k.rows, (int64_t)(blockIdx.x + 1) * rows_per_slab);
  Raw8<A> y, gate;
  Raw8<R> x;
  auto fetch = [&](int64_t r) {
    const int64_t row = i * k.rows + r;
    reader.load(y, row_at<A>(a.y, row) + c);
    reader.load(x, row_at<R>(a.x, row) + c);
    if (rows_gate) reader.load(gate, row_at<A>(a.gate, row) + c);
  };
  int64_t r = blockIdx.x * rows_per_slab + group;
  if (r < r_end) fetch(r);   // (on its way while the parameters are read)
  float g1[8], b1[8], g2[8], b2[8], f[8];
  {
    Raw8<float> p[5];
    const float* const at[5] = {a.p.post_gain, a.p.post_bias, a.p.pre_gain, a.p.pre_bias, k.gate == PBT_GATE_VECTOR ? a.p.gate : nullptr};
#pragma unroll
    for (int q = 0; q < 5; ++q) load_param(reader, p[q], at[q], a.p.stride, i, c);
    get_param(reader, p[0], at[0], 1.f, g1);
    get_param(reader, p[1], at[1], 0.f, b1);
    get_param(reader, p[2], at[2], 1.f, g2);
    get_param(reader, p[3], at[3], 0.f, b2);
    if (k.gate == PBT_GATE_VECTOR) {
      float g[8];
      get_param(reader, p[4], at[4], 0.f, g);
      gate8<false>(k.gate_act, g, f, nullptr);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = 1.f;
    }
  }
  for (; r < r_end; r += ROWS) {
    const int64_t row = i * k.rows + r;
    float u[8], o[8];
    reader.get(y, u);
    reader.get(x, o);
    if (rows_gate) {
      float g[8];
      reader.get(gate, g);
      gate8<false>(k.gate_act, g, f, nullptr);
    }
    if (r + ROWS < r_end) fetch(r + ROWS);   // (on its way while this row is reduced)
    float2 s1 = make_float2(0.f, 1.f), s2 = make_float2(0.f, 1.f);
    if (k.post != PBT_NORM_NONE) {
      s1 = row_stats(u, n, k.post, d, k.eps, sum);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = fmaf(u[e] * s1.y, g1[e], b1[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(k.beta * f[e], u[e], k.alpha * o[e]);
    put8(row_at<R>(a.out, row) + c, o, n);
    if (k.pre != PBT_NORM_NONE) {
      clear_past(o, n);
      s2 = row_stats(o, n, k.pre, d, k.eps, sum);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(o[e] * s2.y, g2[e], b2[e]);
      put8(row_at<A>(a.z, row) + c, o, n);
    }
    if (a.stats && l == 0) reinterpret_cast<float4*>(a.stats)[row] = make_float4(s1.x, s1.y, s2.x, s2.y);
  }
}

template <class A, class R>
void launch(const BlockArgs& a, hipStream_t s) {
  const BlockTeam t = block_team(a.n.d);
  int params = 0;
  for (const float* p : {a.p.post_gain, a.p.post_bias, a.p.pre_gain, a.p.pre_bias, a.p.gate}) params += p ? 1 : 0;
  const int64_t per_slab = block_forward_slab(a.n, params);
  const dim3 grid((unsigned)((a.n.rows + per_slab - 1) / per_slab), a.n.P), block(t.threads);
  if (block_ends_alone(a.n.d)) {
    if (t.T == WIDE) hipLaunchKernelGGL((block_forward_kernel<A, R, WIDE, 1024, true>), grid, block, 0, s, a, per_slab);
    else hipLaunchKernelGGL((block_forward_kernel<A, R, 8, 256, true>), grid, block, 0, s, a, per_slab);
  } else if (t.T == 8) hipLaunchKernelGGL((block_forward_kernel<A, R, 8, 256, false>), grid, block, 0, s, a, per_slab);
  else if (t.T == 32) hipLaunchKernelGGL((block_forward_kernel<A, R, 32, 256, false>), grid, block, 0, s, a, per_slab);
  else if (t.T == 16) hipLaunchKernelGGL((block_forward_kernel<A, R, 16, 256, false>), grid, block, 0, s, a, per_slab);
  else if (t.T == 64) hipLaunchKernelGGL((block_forward_kernel<A, R, 64, 256, false>), grid, block, 0, s, a, per_slab);
  else if (t.threads <= 512) hipLaunchKernelGGL((block_forward_kernel<A, R, WIDE, 512, false>), grid, block, 0, s, a, per_slab);
  else hipLaunchKernelGGL((block_forward_kernel<A, R, WIDE, 1024, false>), grid, block, 0, s, a, per_slab);
}

}  // namespace

hipError_t block_norm_forward(const BlockArgs& a, hipStream_t s) {
  const bool act16 = a.n.dtype == PBT_DTYPE_BF16, res16 = a.n.res_dtype == PBT_DTYPE_BF16;
  if (act16) res16 ? launch<bf16_t, bf16_t>(a, s) : launch<bf16_t, float>(a, s);
  else res16 ? launch<float, bf16_t>(a, s) : launch<float, float>(a, s);
  return hipGetLastError();
}

}  // namespace pbt
