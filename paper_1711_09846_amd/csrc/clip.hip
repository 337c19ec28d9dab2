// The gradient norm of every member over a list of tensors, and clipping: norm_i = sqrt(sum g^2), g <- g max_i / norm_i where norm_i > max_i.
//
// A member's tensors are laid end to end in units of eight elements (a tensor's last unit may be partly empty).  Squares are summed in double: the exact
// square of a float fits, so nothing overflows or vanishes.  Bound by memory: a gradient is read, and where it is clipped read again and written.
//   Small members: one workgroup a member holds the gradient in registers between the sum and the product, so it is read once, in one launch.
//   Larger ones: the units are cut into equal ranges, a workgroup each.  One launch leaves every range's sum; in the next every workgroup adds up its
//   member's sums (the same order everywhere) and scales its range, the ranges that were summed last first: what the cache in front of memory still holds.
// 16 members of 21 million floats (1.34 GB each way): 749 us, three times the gradient at 5.4 TB/s, where a copy, twice the gradient, reaches 5.0; 128 members of
// 202 thousand, which the cache holds: 56 us; 3 members of 6 million bf16 at odd addresses: 26; 8 members of 2372 floats: 3.9 to 4.5.  (Members in batches of half the
// cache, so that every second read is served by it: 882 us for the first of these, the launches are too short to run at the memory's rate.  Vectors moved to
// multiples of 16 bytes: 2 to 7 % slower, an access that crosses a line costs less than the tests.)
#include "operators.h"

namespace pbt {
namespace {

struct ClipTable {
  const char* src[CLIP_TENSORS];
  char* dst[CLIP_TENSORS];
  int64_t len[CLIP_TENSORS], src_stride[CLIP_TENSORS], dst_stride[CLIP_TENSORS];   // elements
  int64_t start[CLIP_TENSORS + 1];   // first unit of every tensor
  uint64_t bf16;                     // bit k: tensor k is bf16
  int n;
};
constexpr int TABLE_WORDS = 5 * CLIP_TENSORS + CLIP_TENSORS + 1;
static_assert(sizeof(ClipTable) == (TABLE_WORDS + 2) * 8, "the table is copied word by word");

// where a thread looks a unit's tensor up: the table's columns, in LDS
struct Lookup {
  const uint64_t* w;
  int n;
  uint64_t bf16;
  __device__ __forceinline__ int64_t start(int k) const { return (int64_t)w[5 * CLIP_TENSORS + k]; }
  __device__ __forceinline__ int of(int64_t u) const {
    int lo = 0, hi = n;   // start(lo) <= u < start(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start(mid) <= u) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};
__device__ __forceinline__ Lookup copy_table(const ClipTable& t, uint64_t* lds) {
  const uint64_t* words = reinterpret_cast<const uint64_t*>(&t);
  for (int k = threadIdx.x; k < TABLE_WORDS; k += blockDim.x) lds[k] = words[k];
  __syncthreads();
  return Lookup{lds, t.n, t.bf16};
}

// a unit as it lies in memory
struct Unit8 { Vec16 a, b; };
__device__ __forceinline__ void unpack(const Unit8& u, bool half, float* v) {
  if (half) {
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[2 * q] = __uint_as_float(u.a.w[q] << 16); v[2 * q + 1] = __uint_as_float(u.a.w[q] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[q] = __uint_as_float(u.a.w[q]); v[4 + q] = __uint_as_float(u.b.w[q]); }
  }
}
struct Place { const char* src; char* dst; int n; bool half; };   // of a unit: its addresses and how many of its elements exist
__device__ __forceinline__ Place place(const Lookup& t, int member, int64_t u) {
  const int k = t.n > 1 ? t.of(u) : 0;
  const int64_t e = (u - t.start(k)) * 8, left = (int64_t)t.w[2 * CLIP_TENSORS + k] - e;
  const bool half = (t.bf16 >> k) & 1;
  const int shift = half ? 1 : 2;
  return Place{reinterpret_cast<const char*>(t.w[k]) + ((member * (int64_t)t.w[3 * CLIP_TENSORS + k] + e) << shift),
               reinterpret_cast<char*>(t.w[CLIP_TENSORS + k]) + ((member * (int64_t)t.w[4 * CLIP_TENSORS + k] + e) << shift), left < 8 ? (int)left : 8, half};
}
__device__ __forceinline__ Unit8 read(const Place& p) {
  Unit8 u;
  u.b = Vec16{{0, 0, 0, 0}};
  if (p.half) {
    Raw8<bf16_t> r;
    r.load(reinterpret_cast<const bf16_t*>(p.src), p.n);
    u.a = r.a;
  } else {
    Raw8<float> r;
    r.load(reinterpret_cast<const float*>(p.src), p.n);
    u.a = r.a;
    u.b = r.b;
  }
  return u;
}
__device__ __forceinline__ void write(const Place& p, const float* v) {
  if (p.half) put8(reinterpret_cast<bf16_t*>(p.dst), v, p.n);
  else put8(reinterpret_cast<float*>(p.dst), v, p.n);
}
__device__ __forceinline__ double squares(const float* v, double acc) {
#pragma unroll
  for (int q = 0; q < 8; ++q) acc = fma((double)v[q], (double)v[q], acc);
  return acc;
}

template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) t += red[w];
  return t;
}
// the factor of a member of norm n; 1: it stays as it is.  (Rounded to float once, like the norm that is handed out.)
__device__ __forceinline__ float factor(double n, const float* max_norm) {
  double m = (double)*max_norm;
  m = m < 0.0 ? 0.0 : m;   // (NaN stays: no comparison with it holds)
  return n > m ? (float)(m / n) : 1.f;
}

// ---- small members: held in registers ----
// PER units a thread.  (More of them would leave a compute unit one workgroup: 1024 members of 20000 floats take 31 us with 4, 49 with 8.)
template <int PER>
__global__ __launch_bounds__(CLIP_HELD_THREADS) void clip_held_kernel(ClipTable table, const float* __restrict__ max_norm, int64_t max_norm_stride, float* __restrict__ norm) {
  __shared__ uint64_t words[TABLE_WORDS];
  __shared__ double red[CLIP_HELD_THREADS / 64];
  const int i = blockIdx.x;
  const Lookup t = copy_table(table, words);
  const int64_t total = t.start(t.n);
  Unit8 u[PER];
  uint32_t half = 0;   // bit j: unit j is bf16
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t at = threadIdx.x + j * CLIP_HELD_THREADS;
    u[j] = Unit8{};
    if (at < total) {
      const Place p = place(t, i, at);
      u[j] = read(p);
      half |= p.half ? 1u << j : 0u;
    }
  }
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (threadIdx.x + j * CLIP_HELD_THREADS < total) {
      float v[8];
      unpack(u[j], (half >> j) & 1, v);
      s = squares(v, s);
    }
  const double n = sqrt(block_sum<CLIP_HELD_THREADS>(s, red));
  if (norm && threadIdx.x == 0) norm[i] = (float)n;
  if (!max_norm) return;
  const float c = factor(n, max_norm + i * max_norm_stride);
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t at = threadIdx.x + j * CLIP_HELD_THREADS;
    if (at >= total) break;
    const Place p = place(t, i, at);
    if (c == 1.f && p.src == p.dst) continue;
    float v[8];
    unpack(u[j], p.half, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= c;
    write(p, v);
  }
}

// ---- large members: ranges ----
// The units [lo, hi) of one tensor as 16-byte vectors, adjacent threads on adjacent vectors, DEEP of them requested at a time; the elements of a last unit that is
// not whole one by one.  SCALE: dst = c src, NT past the caches; else the sum of squares is returned.
constexpr int DEEP = 4;
template <class T, bool SCALE, bool NT>
__device__ __forceinline__ double along_tensor(const T* src, T* dst, int64_t len, int64_t lo, int64_t hi, float c) {
  constexpr int V = 16 / (int)sizeof(T);   // elements of a vector
  double acc = 0.0;
  auto use = [&](Vec16 x, int64_t at) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (V == 8) {
        float a = __uint_as_float(x.w[q] << 16), b = __uint_as_float(x.w[q] & 0xffff0000u);
        if (SCALE) x.w[q] = f2bf_pair(a * c, b * c);
        else acc = fma((double)b, (double)b, fma((double)a, (double)a, acc));
      } else {
        const float a = __uint_as_float(x.w[q]);
        if (SCALE) x.w[q] = __float_as_uint(a * c);
        else acc = fma((double)a, (double)a, acc);
      }
    }
    if (SCALE) {
      if (NT) stream16(dst + at * V, x);
      else store16(dst + at * V, x);
    }
  };
  const int64_t end = min(hi, len / 8) * (8 / V);
  int64_t at = lo * (8 / V) + threadIdx.x;
  for (; at + (DEEP - 1) * 256 < end; at += DEEP * 256) {
    Vec16 x[DEEP];
#pragma unroll
    for (int q = 0; q < DEEP; ++q) x[q] = load16(src + (at + q * 256) * V);
#pragma unroll
    for (int q = 0; q < DEEP; ++q) use(x[q], at + q * 256);
  }
  for (; at < end; at += 256) use(load16(src + at * V), at);
  if (hi * 8 > len && threadIdx.x < len % 8) {   // (the range holds the tensor's end)
    const int64_t e = len / 8 * 8 + threadIdx.x;
    const float v = V == 8 ? bf2f((bf16_t)src[e]) : (float)src[e];
    if (!SCALE) acc = fma((double)v, (double)v, acc);
    else if (V == 8) dst[e] = (T)f2bf(v * c);
    else dst[e] = (T)(v * c);
  }
  return acc;
}

// the units [lo, hi) of a member: tensor by tensor where the range's tensors are long enough to keep the workgroup busy, else unit by unit
template <bool SCALE, bool NT>
__device__ __forceinline__ double walk(const ClipTable& t, uint64_t* words, int member, int64_t lo, int64_t hi, float c) {
  double acc = 0.0;
  if (lo >= hi) return acc;
  // the tensors of the range, by a vote of lanes that look at one tensor each (a loop over the table costs a scalar load after another)
  const int lane = threadIdx.x & 63;
  const int64_t start = lane < t.n ? t.start[lane] : INT64_MAX;
  const int first = __popcll(__ballot(start <= lo)) - 1, last = __popcll(__ballot(start < hi)) - 1;
  if ((int64_t)(last - first) * 512 <= hi - lo) {   // (4 members with 110 tensors of 100 to 4133 floats: 24 us so, 28 tensor by tensor)
    for (int k = first; k <= last; ++k) {
      const int64_t a = max(lo, t.start[k]) - t.start[k], b = min(hi, t.start[k + 1]) - t.start[k];
      const int64_t from = member * t.src_stride[k], to = member * t.dst_stride[k];
      if ((t.bf16 >> k) & 1)
        acc += along_tensor<bf16_t, SCALE, NT>(reinterpret_cast<const bf16_t*>(t.src[k]) + from, reinterpret_cast<bf16_t*>(t.dst[k]) + to, t.len[k], a, b, c);
      else
        acc += along_tensor<float, SCALE, NT>(reinterpret_cast<const float*>(t.src[k]) + from, reinterpret_cast<float*>(t.dst[k]) + to, t.len[k], a, b, c);
    }
    return acc;
  }
  const Lookup l = copy_table(t, words);
  for (int64_t u = lo + threadIdx.x; u < hi; u += 256) {
    const Place p = place(l, member, u);
    float v[8];
    unpack(read(p), p.half, v);
    if (SCALE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= c;
      write(p, v);
    } else {
      acc = squares(v, acc);
    }
  }
  return acc;
}

__global__ __launch_bounds__(256) void clip_sum_kernel(ClipTable t, int64_t per_range, double* __restrict__ part, int64_t n_part, int64_t first) {
  __shared__ uint64_t words[TABLE_WORDS];
  __shared__ double red[4];
  const int i = blockIdx.y;
  const int64_t lo = (int64_t)blockIdx.x * per_range, hi = min(lo + per_range, t.start[t.n]);
  const double s = block_sum<256>(walk<false, false>(t, words, i, lo, hi, 0.f), red);
  if (threadIdx.x == 0) part[i * n_part + first + blockIdx.x] = s;
}

// write_norm: the first range's workgroup hands the norm out; max_norm = null: only that.  The ranges that were summed last are taken first.
template <bool NT>
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipTable t, int64_t per_range, const double* __restrict__ part, int64_t n_part,
                                                         const float* __restrict__ max_norm, int64_t max_norm_stride, float* __restrict__ norm, int in_place) {
  __shared__ uint64_t words[TABLE_WORDS];
  __shared__ double red[4];
  const int i = gridDim.y - 1 - blockIdx.y;
  const int64_t range = gridDim.x - 1 - blockIdx.x;
  double s = 0.0;
  for (int64_t k = threadIdx.x; k < n_part; k += 256) s += part[i * n_part + k];
  const double n = sqrt(block_sum<256>(s, red));
  if (norm && range == 0 && threadIdx.x == 0) norm[i] = (float)n;
  if (!max_norm) return;
  const float c = factor(n, max_norm + i * max_norm_stride);
  if (c == 1.f && in_place) return;
  const int64_t lo = range * per_range, hi = min(lo + per_range, t.start[t.n]);
  walk<true, NT>(t, words, i, lo, hi, c);
}

// norm and factor of a member from its ranges' sums
__global__ __launch_bounds__(256) void clip_factor_kernel(const double* __restrict__ part, int64_t n_part, const float* __restrict__ max_norm, int64_t max_norm_stride,
                                                          float* __restrict__ norm, float* __restrict__ out) {
  __shared__ double red[4];
  const int i = blockIdx.x;
  double s = 0.0;
  for (int64_t k = threadIdx.x; k < n_part; k += 256) s += part[i * n_part + k];
  const double n = sqrt(block_sum<256>(s, red));
  if (threadIdx.x == 0) {
    norm[i] = (float)n;
    out[i] = factor(n, max_norm + i * max_norm_stride);
  }
}

ClipTable table(const pbt_grad* g, int k0, int n, bool* in_place) {
  ClipTable t;
  t.n = std::min(n - k0, CLIP_TENSORS);
  t.bf16 = 0;
  *in_place = true;
  int64_t at = 0;
  for (int k = 0; k < t.n; ++k) {
    const pbt_grad& e = g[k0 + k];
    t.src[k] = static_cast<const char*>(e.d_src);
    t.dst[k] = static_cast<char*>(e.d_dst);
    t.len[k] = e.len; t.src_stride[k] = e.src_stride; t.dst_stride[k] = e.dst_stride;
    t.start[k] = at;
    at += clip_units(e);
    if (e.dtype == PBT_DTYPE_BF16) t.bf16 |= 1ull << k;
    if (e.d_src != e.d_dst) *in_place = false;
  }
  t.start[t.n] = at;
  for (int k = t.n; k < CLIP_TENSORS; ++k) {
    t.src[k] = nullptr; t.dst[k] = nullptr;
    t.len[k] = t.src_stride[k] = t.dst_stride[k] = 0;
    t.start[k + 1] = at;
  }
  return t;
}

}  // namespace

size_t clip_work_bytes(const pbt_grad* g, int n, int P) { return (size_t)P * clip_parts(g, n, P) * sizeof(double); }

size_t grad_factor_work_bytes(int64_t stride, int P) {
  const pbt_grad g{nullptr, nullptr, stride, stride, stride, PBT_DTYPE_FP32, 0};
  return (size_t)P * clip_parts(&g, 1, P) * sizeof(double);
}
hipError_t grad_factor(const float* G, int64_t stride, int P, const float* max_norm, int64_t max_norm_stride, float* norm, float* out, void* work, hipStream_t s) {
  const pbt_grad g{G, nullptr, stride, stride, stride, PBT_DTYPE_FP32, 0};
  bool in_place;
  const ClipTable t = table(&g, 0, 1, &in_place);
  const int64_t total = t.start[1], ranges = clip_sum_ranges(total, P), per_range = (total + ranges - 1) / ranges;
  double* part = static_cast<double*>(work);
  hipLaunchKernelGGL(clip_sum_kernel, dim3((unsigned)ranges, P), dim3(256), 0, s, t, per_range, part, ranges, (int64_t)0);
  hipLaunchKernelGGL(clip_factor_kernel, dim3(P), dim3(256), 0, s, part, ranges, max_norm, max_norm_stride, norm, out);
  return hipGetLastError();
}

hipError_t clip_gradients(const pbt_grad* g, int n, int P, const float* max_norm, int64_t max_norm_stride, float* norm, void* work, hipStream_t s) {
  bool in_place;
  if (const int per = clip_held(g, n, P)) {
    const ClipTable t = table(g, 0, n, &in_place);
    if (per == 4) hipLaunchKernelGGL(clip_held_kernel<4>, dim3(P), dim3(CLIP_HELD_THREADS), 0, s, t, max_norm, max_norm_stride, norm);
    else hipLaunchKernelGGL(clip_held_kernel<8>, dim3(P), dim3(CLIP_HELD_THREADS), 0, s, t, max_norm, max_norm_stride, norm);
    return hipGetLastError();
  }
  double* part = static_cast<double*>(work);
  const int64_t n_part = clip_parts(g, n, P);
  int64_t bytes = 0;
  for (int k = 0; k < n; ++k) bytes += P * g[k].len * (g[k].dtype == PBT_DTYPE_BF16 ? 2 : 4);
  for (int pass = 0; pass < 2; ++pass) {
    int64_t first = 0;
    for (int k0 = 0; k0 < n; k0 += CLIP_TENSORS) {
      const ClipTable t = table(g, k0, n, &in_place);
      const int64_t total = t.start[t.n], ranges = pass == 0 ? clip_sum_ranges(total, P) : max_norm ? clip_scale_ranges(total, P) : 1, per_range = (total + ranges - 1) / ranges;
      const dim3 grid((unsigned)ranges, P);
      if (pass == 0)
        hipLaunchKernelGGL(clip_sum_kernel, grid, dim3(256), 0, s, t, per_range, part, n_part, first);
      else if (!max_norm && k0 > 0)
        break;
      else if (clip_past_caches(bytes))
        hipLaunchKernelGGL(clip_scale_kernel<true>, grid, dim3(256), 0, s, t, per_range, part, n_part, max_norm, max_norm_stride, k0 == 0 ? norm : nullptr, (int)in_place);
      else
        hipLaunchKernelGGL(clip_scale_kernel<false>, grid, dim3(256), 0, s, t, per_range, part, n_part, max_norm, max_norm_stride, k0 == 0 ? norm : nullptr, (int)in_place);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      first += ranges;
    }
  }
  return hipSuccess;
}

}  // namespace pbt
