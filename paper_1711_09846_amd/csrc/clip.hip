// The gradient norm of every member over a list of tensors, and clipping: norm_i = sqrt(sum g^2), g <- g max_i / norm_i where norm_i > max_i.
//
// A member's tensors are laid end to end in units of eight elements (a tensor's last unit may be partly empty), and the units are cut into equal ranges, one
// workgroup each.  Two launches: partial sums of squares of every range, then every workgroup adds up its member's partial sums (the same order
// everywhere) and scales its range.  Squares are summed in double: the exact square of a float fits, so nothing overflows or vanishes, and the
// order, fixed, does not show.
#include "operators.h"

namespace pbt {
namespace {

constexpr int CLIP_TENSORS = 64;   // of one launch (the table is a kernel argument)
struct ClipTable {
  const char* src[CLIP_TENSORS];
  char* dst[CLIP_TENSORS];
  int64_t len[CLIP_TENSORS], src_stride[CLIP_TENSORS], dst_stride[CLIP_TENSORS];   // elements
  int64_t start[CLIP_TENSORS + 1];   // first unit of every tensor
  uint64_t bf16;                     // bit k: tensor k is bf16
  int n;
  int64_t per_chunk;                 // units of a range
};

__device__ __forceinline__ int tensor_of(const int64_t* start, int n, int64_t u) {
  int lo = 0, hi = n;   // start[lo] <= u < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= u) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) t += red[w];
  __syncthreads();
  return t;
}

template <bool SCALE>
__device__ __forceinline__ double walk(const ClipTable& t, int member, int64_t lo, int64_t hi, float c) {
  double acc = 0.0;
  for (int64_t u = lo + threadIdx.x; u < hi; u += blockDim.x) {
    const int k = tensor_of(t.start, t.n, u);
    const int64_t e = (u - t.start[k]) * 8;
    const int64_t left = t.len[k] - e;
    const int n = left < 8 ? (int)left : 8;
    float v[8];
    const bool half = (t.bf16 >> k) & 1;
    if (half) {
      Raw8<bf16_t> r;
      r.load(reinterpret_cast<const bf16_t*>(t.src[k]) + member * t.src_stride[k] + e, n);
      r.get(v);
    } else {
      Raw8<float> r;
      r.load(reinterpret_cast<const float*>(t.src[k]) + member * t.src_stride[k] + e, n);
      r.get(v);
    }
    if (!SCALE) {
#pragma unroll
      for (int q = 0; q < 8; ++q) acc = fma((double)v[q], (double)v[q], acc);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] *= c;
      if (half) put8(reinterpret_cast<bf16_t*>(t.dst[k]) + member * t.dst_stride[k] + e, v, n);
      else put8(reinterpret_cast<float*>(t.dst[k]) + member * t.dst_stride[k] + e, v, n);
    }
  }
  return acc;
}

__global__ __launch_bounds__(256) void clip_sum_kernel(ClipTable t, double* __restrict__ part, int64_t part_stride, int64_t first) {
  __shared__ double red[4];
  const int64_t lo = (int64_t)blockIdx.x * t.per_chunk, hi = min(lo + t.per_chunk, t.start[t.n]);
  const double s = block_sum(walk<false>(t, blockIdx.y, lo, hi, 0.f), red);
  if (threadIdx.x == 0) part[blockIdx.y * part_stride + first + blockIdx.x] = s;
}

// chunk 0 of the first launch writes the norm; max_norm = null: only that
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipTable t, const double* __restrict__ part, int64_t n_part, const float* __restrict__ max_norm,
                                                         int64_t max_norm_stride, float* __restrict__ norm, int write_norm, uint64_t in_place) {
  __shared__ double red[4];
  const int i = blockIdx.y;
  double s = 0.0;
  for (int64_t k = threadIdx.x; k < n_part; k += 256) s += part[i * n_part + k];
  const double n = sqrt(block_sum(s, red));
  if (write_norm && norm && blockIdx.x == 0 && threadIdx.x == 0) norm[i] = (float)n;
  if (!max_norm) return;
  const double m = (double)max_norm[i * max_norm_stride];
  const float c = n > m ? (float)(fmax(m, 0.0) / n) : 1.f;
  const int64_t lo = (int64_t)blockIdx.x * t.per_chunk, hi = min(lo + t.per_chunk, t.start[t.n]);
  if (!(n > m) && in_place) return;
  walk<true>(t, i, lo, hi, c);
}

int64_t units(const pbt_grad& g) { return (g.len + 7) / 8; }
// ranges of a launch over `total` units per member
int64_t chunks_of(int64_t total, int P) {
  int64_t most = 4096 / P;
  if (most < 1) most = 1;
  const int64_t by_size = (total + 255) / 256;   // at least a unit per thread
  const int64_t c = by_size < most ? by_size : most;
  return c < 1 ? 1 : c;
}
int64_t parts(const pbt_grad* g, int n, int P) {
  int64_t sum = 0;
  for (int k0 = 0; k0 < n; k0 += CLIP_TENSORS) {
    int64_t total = 0;
    for (int k = k0; k < n && k < k0 + CLIP_TENSORS; ++k) total += units(g[k]);
    sum += chunks_of(total, P);
  }
  return sum;
}
ClipTable table(const pbt_grad* g, int k0, int n, int64_t* total, bool* in_place) {
  ClipTable t;
  t.n = n - k0 < CLIP_TENSORS ? n - k0 : CLIP_TENSORS;
  t.bf16 = 0;
  *in_place = true;
  int64_t at = 0;
  for (int k = 0; k < t.n; ++k) {
    const pbt_grad& e = g[k0 + k];
    t.src[k] = static_cast<const char*>(e.d_src);
    t.dst[k] = static_cast<char*>(e.d_dst);
    t.len[k] = e.len; t.src_stride[k] = e.src_stride; t.dst_stride[k] = e.dst_stride;
    t.start[k] = at;
    at += units(e);
    if (e.dtype == PBT_DTYPE_BF16) t.bf16 |= 1ull << k;
    if (e.d_src != e.d_dst) *in_place = false;
  }
  t.start[t.n] = at;
  *total = at;
  return t;
}

}  // namespace

size_t clip_work_bytes(const pbt_grad* g, int n, int P) { return (size_t)P * parts(g, n, P) * sizeof(double); }

hipError_t clip_gradients(const pbt_grad* g, int n, int P, const float* max_norm, int64_t max_norm_stride, float* norm, void* work, hipStream_t s) {
  double* part = static_cast<double*>(work);
  const int64_t n_part = parts(g, n, P);
  for (int pass = 0; pass < 2; ++pass) {
    int64_t first = 0;
    for (int k0 = 0; k0 < n; k0 += CLIP_TENSORS) {
      int64_t total;
      bool in_place;
      ClipTable t = table(g, k0, n, &total, &in_place);
      const int64_t chunks = chunks_of(total, P);
      t.per_chunk = (total + chunks - 1) / chunks;
      if (pass == 0)
        hipLaunchKernelGGL(clip_sum_kernel, dim3((unsigned)chunks, P), dim3(256), 0, s, t, part, n_part, first);
      else if (max_norm || k0 == 0)
        hipLaunchKernelGGL(clip_scale_kernel, dim3(max_norm ? (unsigned)chunks : 1u, P), dim3(256), 0, s, t, part, n_part, max_norm, max_norm_stride, norm,
                           k0 == 0, in_place);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      first += chunks;
    }
  }
  return hipSuccess;
}

}  // namespace pbt
