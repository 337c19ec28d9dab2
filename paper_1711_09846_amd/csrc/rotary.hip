// Rotary positions: pair j of a head at position p is turned by p f_j.
//
// Bound by memory: every element is read and written once.  The angles are what could be in the way: their sine and cosine take some sixty instructions, as
// much as moving a pair takes at the memory's rate, so a workgroup forms them once for a few rows, in LDS, and all heads of those rows use them.  A unit of
// work is one 16-byte access of adjacent pairs (two where a pair's halves lie apart), one a thread and sweep: with four on their way in a thread's registers
// fewer workgroups fit a compute unit (131072 rows: 812 us).
// 16 of 24 heads of 64 in 65536 rows, bf16: 53 us, a copy of the same heads 49; 40 of 60 heads of 128 in 131072 rows: 491 us (5.5 TB/s), a copy 472; fp32 rows
// of 5 heads of 84 with 42 turned, 9973 of them: 9.5 us, a copy 6.8; 16 rows: 3.0.  A group of heads forms its own angles: 32 heads of 128 in 16384 rows take 41 us
// in place, one key head in the same call 5 us more (by its bytes 1.3); 50000 rows of one head of 128: 13 us (1.9 TB/s).
#include <cmath>

#include "operators.h"

namespace pbt {
namespace {

__global__ __launch_bounds__(256) void rotary_plan_kernel(RotaryFrequencies f, int n, double* __restrict__ table) {
  if ((int)threadIdx.x < n) table[threadIdx.x] = f.turns[threadIdx.x];
}

// cos and sin of p f, given in turns: the product and the reduction to a quarter turn in double (at position 2^31 the product is good to 1e-7 of a turn, at a
// million to 1e-10), what is left, x within +-pi/4, in float by the Taylor series: x^11 / 11! and x^12 / 12! are below 2e-9
__device__ __forceinline__ float2 turn(double turns) {
  const double quarters = 4.0 * turns, q = rint(quarters);
  const float x = (float)(quarters - q) * 1.57079632679489662f;
  const int k = (int)fma(-4.0, floor(0.25 * q), q);   // q mod 4
  const float y = x * x;
  const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -0.166666667f), x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.f);
  const float a = (k & 1) ? s : c, b = (k & 1) ? c : s;   // quarter turns: (c, s), (-s, c), (-c, -s), (s, -c)
  return make_float2(k == 1 || k == 2 ? -a : a, k >= 2 ? -b : b);
}

__device__ __forceinline__ int64_t position(const RotaryArgs& a, int64_t row) {
  if (a.pos) return a.pos64 ? static_cast<const int64_t*>(a.pos)[row] : (int64_t)static_cast<const int32_t*>(a.pos)[row];
  return a.start + (a.period > 0 ? (int64_t)((uint32_t)row % (uint32_t)a.period) : row);   // (rows and period are below 2^31)
}

// 16 bytes of elements, or the n < V that there are
template <class T> struct Unit;
template <> struct Unit<bf16_t> {
  static constexpr int V = 8;
  static __device__ __forceinline__ Vec16 load(const bf16_t* p, int n) { Raw8<bf16_t> r; r.load(p, n); return r.a; }
  // the elements of a word, and back
  static __device__ __forceinline__ void get(uint32_t w, float* v) { v[0] = __uint_as_float(w << 16); v[1] = __uint_as_float(w & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t make(const float* v) { return f2bf_pair(v[0], v[1]); }
  static __device__ __forceinline__ void store_some(bf16_t* p, const Vec16& a, int n) {
#pragma unroll
    for (int e = 0; e < V - 1; ++e)
      if (e < n) p[e] = (bf16_t)(a.w[e >> 1] >> (16 * (e & 1)));
  }
};
template <> struct Unit<float> {
  static constexpr int V = 4;
  static __device__ __forceinline__ Vec16 load(const float* p, int n) {
    if (n >= V) return load16(p);
    Vec16 a{{0, 0, 0, 0}};
#pragma unroll
    for (int e = 0; e < V - 1; ++e)
      if (e < n) a.w[e] = __float_as_uint(p[e]);
    return a;
  }
  static __device__ __forceinline__ void get(uint32_t w, float* v) { v[0] = __uint_as_float(w); }
  static __device__ __forceinline__ uint32_t make(const float* v) { return __float_as_uint(v[0]); }
  static __device__ __forceinline__ void store_some(float* p, const Vec16& a, int n) {
#pragma unroll
    for (int e = 0; e < V - 1; ++e)
      if (e < n) p[e] = __uint_as_float(a.w[e]);
  }
};

template <class T, bool NT>
__device__ __forceinline__ void put(T* p, const Vec16& a, int n) {
  if (n < Unit<T>::V) Unit<T>::store_some(p, a, n);
  else if (NT) stream16(p, a);
  else store16(p, a);
}

// n / d for n d < 2^32, by a product with ceil(2^32 / d) (d = 1: 0)
__device__ __forceinline__ int quotient(int n, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)n, magic) : n; }

// NT: stores that no cache keeps
template <class T, int LAYOUT, bool NT>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, RotaryShapes shapes, int pitch) {
  extern __shared__ float table[];   // [rows][pitch] cosines, then sines
  constexpr int V = Unit<T>::V;
  constexpr int PV = rotary_unit_pairs(V, LAYOUT == PBT_ROTARY_HALF);
  // the workgroup's group of heads (one after the other in the grid)
  RotaryShape w = shapes.g[0];
  pbt_heads grp = a.g[0];
  int64_t block = blockIdx.x;
#pragma unroll
  for (int g = 1; g < 4; ++g)
    if (g < a.n_groups && block >= w.blocks) {
      block -= w.blocks;
      w = shapes.g[g];
      grp = a.g[g];
    }
  const int pairs = a.rot / 2, head0 = (int)((uint32_t)block % (uint32_t)w.head_blocks) * w.heads, heads = min(w.heads, grp.heads - head0);
  // Where results go elsewhere, a last unit that would not be whole starts earlier instead: what it shares with its neighbour both compute alike.  (In
  // place one of the two could read what the other has written.)
  const bool apart = grp.d_src != grp.d_dst, pairs_back = apart && pairs >= PV, copy_back = a.width - a.rot >= V;
  struct Item { const T* src; T* dst; Vec16 x, y; int lds, n; };   // n: pairs (-elements where the unit is copied); lds: the unit's first angle
  for (int64_t row0 = (int64_t)((uint32_t)block / (uint32_t)w.head_blocks) * w.rows; row0 < a.rows; row0 += (int64_t)w.row_blocks * w.rows) {
    const int rows = (int)min((int64_t)w.rows, a.rows - row0);
    // (a workgroup's last block of heads may be short: items are counted over w.heads and those past the end skipped)
    const int items = rows * w.heads * w.units;
    auto fetch = [&](int k) {
      Item it;
      it.n = 0;
      if (k >= items) return it;
      const int q = quotient(k, w.by_units), u = k - q * w.units, r = quotient(q, w.by_heads);
      const int h = q - r * w.heads;
      if (h >= heads) return it;
      it.src = static_cast<const T*>(grp.d_src) + (row0 + r) * grp.src_row + (head0 + h) * grp.src_head;
      it.dst = static_cast<T*>(grp.d_dst) + (row0 + r) * grp.dst_row + (head0 + h) * grp.dst_head;
      if (u < w.pair_units) {
        const int j = pairs_back ? min(u * PV, pairs - PV) : u * PV;
        it.n = min(PV, pairs - j);
        it.lds = r * pitch + j;
        if (LAYOUT == PBT_ROTARY_HALF) {
          it.src += j;
          it.dst += j;
          it.x = Unit<T>::load(it.src, it.n);
          it.y = Unit<T>::load(it.src + pairs, it.n);
        } else {
          it.src += 2 * j;
          it.dst += 2 * j;
          it.x = Unit<T>::load(it.src, 2 * it.n);
        }
      } else {
        const int from = a.rot + (u - w.pair_units) * V, e = copy_back ? min(from, a.width - V) : from;
        it.src += e;
        it.dst += e;
        it.n = -min(V, a.width - e);
        it.x = Unit<T>::load(it.src, -it.n);
      }
      return it;
    };
    Item it = fetch(threadIdx.x);   // (on its way while the angles are formed)
    for (int k = threadIdx.x; k < rows * pitch; k += 256) {
      const int r = quotient(k, w.by_pitch), j = k - r * pitch;
      if (j < pairs) {
        const float2 cs = turn((double)position(a, row0 + r) * a.turns[j]);
        table[k] = cs.x * a.gain;
        table[w.rows * pitch + k] = cs.y * a.gain * a.sign;
      }
    }
    __syncthreads();
    for (int k = threadIdx.x;;) {
      if (it.n < 0) {
        put<T, NT>(it.dst, it.x, -it.n);
      } else if (it.n > 0) {
        // (word by word, so that few angles are in registers at a time)
        const float *c = table + it.lds, *s = c + w.rows * pitch;
        constexpr int WE = V / 4;   // elements of a word
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[2], y[2];
          Unit<T>::get(it.x.w[q], x);
          if (LAYOUT == PBT_ROTARY_HALF) {
            Unit<T>::get(it.y.w[q], y);
#pragma unroll
            for (int e = 0; e < WE; ++e) {
              const float u = x[e], v = y[e], ce = c[q * WE + e], se = s[q * WE + e];
              x[e] = u * ce - v * se;
              y[e] = v * ce + u * se;
            }
            it.y.w[q] = Unit<T>::make(y);
          } else if (WE == 2) {
            const float u = x[0], v = x[1], ce = c[q], se = s[q];
            x[0] = u * ce - v * se;
            x[1] = v * ce + u * se;
          } else if (q & 1) {
            const float u = __uint_as_float(it.x.w[q - 1]), v = x[0], ce = c[q / 2], se = s[q / 2];
            it.x.w[q - 1] = __float_as_uint(u * ce - v * se);
            x[0] = v * ce + u * se;
          }
          it.x.w[q] = Unit<T>::make(x);
        }
        if (LAYOUT == PBT_ROTARY_HALF) {
          put<T, NT>(it.dst, it.x, it.n);
          put<T, NT>(it.dst + pairs, it.y, it.n);
        } else {
          put<T, NT>(it.dst, it.x, 2 * it.n);
        }
      }
      k += 256;
      if (k - (int)threadIdx.x >= items) break;
      it = fetch(k);
    }
    __syncthreads();   // (the table is written again)
  }
}

template <class T, int LAYOUT>
hipError_t launch(RotaryArgs a, hipStream_t s) {
  if (a.period >= a.rows) a.period = 0;   // (the rows end before it does)
  RotaryCall call{Unit<T>::V, LAYOUT == PBT_ROTARY_HALF, a.rot, a.width, a.rows, a.n_groups, {}, {}};
  for (int g = 0; g < a.n_groups; ++g) {
    call.heads[g] = a.g[g].heads;
    call.apart[g] = a.g[g].d_src != a.g[g].d_dst;
  }
  const RotaryCut cut = rotary_cut(call);
  const size_t lds = (size_t)cut.table * sizeof(float);
  int64_t bytes = 0;
  for (int g = 0; g < a.n_groups; ++g) bytes += a.rows * a.g[g].heads * a.width * (int64_t)sizeof(T);
  if (rotary_past_caches(bytes)) hipLaunchKernelGGL((rotary_kernel<T, LAYOUT, true>), dim3((unsigned)cut.blocks), dim3(256), lds, s, a, cut.shapes, cut.pitch);
  else hipLaunchKernelGGL((rotary_kernel<T, LAYOUT, false>), dim3((unsigned)cut.blocks), dim3(256), lds, s, a, cut.shapes, cut.pitch);
  return hipGetLastError();
}

}  // namespace

void rotary_frequencies(const pbt_rotary& r, RotaryFrequencies* f) {
  const double two_pi = 6.283185307179586476925;
  const double base = r.scaling == PBT_ROTARY_SCALE_BASE && r.rot_dim > 2 ? r.base * std::pow(r.factor, r.rot_dim / (r.rot_dim - 2.0)) : r.base;
  for (int j = 0; j < PBT_ROTARY_MAX_DIM / 2; ++j) {
    f->turns[j] = 0.0;
    if (j >= r.rot_dim / 2) continue;
    double w = std::isfinite(base) ? std::pow(base, -2.0 * j / r.rot_dim) : base;   // radians a position (no base: none)
    if (r.scaling == PBT_ROTARY_SCALE_LINEAR) w /= r.factor;
    if (r.scaling == PBT_ROTARY_SCALE_RAMP) {
      const double at = (r.trained_len * w / two_pi - r.low) / (r.high - r.low), keep = at < 0.0 ? 0.0 : at > 1.0 ? 1.0 : at;
      w *= keep + (1.0 - keep) / r.factor;
    }
    f->turns[j] = w / two_pi;
  }
}

hipError_t rotary_plan(const RotaryFrequencies& f, int n, double* table, hipStream_t s) {
  hipLaunchKernelGGL(rotary_plan_kernel, dim3(1), dim3(256), 0, s, f, n, table);
  return hipGetLastError();
}

hipError_t rotary_apply(const RotaryArgs& a, int layout, int dtype, hipStream_t s) {
  if (dtype == PBT_DTYPE_BF16) return layout == PBT_ROTARY_HALF ? launch<bf16_t, PBT_ROTARY_HALF>(a, s) : launch<bf16_t, PBT_ROTARY_INTERLEAVED>(a, s);
  return layout == PBT_ROTARY_HALF ? launch<float, PBT_ROTARY_HALF>(a, s) : launch<float, PBT_ROTARY_INTERLEAVED>(a, s);
}

}  // namespace pbt
