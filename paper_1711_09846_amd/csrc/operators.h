// Launchers behind the operators of include/pbt.h that need no handle (clip.hip, rotary.hip, block_norm_forward.hip, block_norm_backward.hip), and what their kernels share: groups of
// eight elements of either type at any address.  Every launcher only enqueues on `s`; arguments have been checked by the entry points.
#pragma once
#include <type_traits>

#include "common.h"
#include "operators_choose.h"
#include "../../include/pbt.h"

namespace pbt {

// ---- eight consecutive elements at an address that is a multiple of the element's size only ----
// (global memory takes 16-byte accesses at any address: the compiler emits one for these copies, and where the address is a multiple of 16 they cost
// what an aligned access costs)
struct Vec16 { uint32_t w[4]; };
__device__ __forceinline__ Vec16 load16(const void* p) { Vec16 v; __builtin_memcpy(&v, p, 16); return v; }
__device__ __forceinline__ void store16(void* p, const Vec16& v) { __builtin_memcpy(p, &v, 16); }
// the same past the caches
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void stream16(void* p, const Vec16& v) {
  const u32x4_any x = {v.w[0], v.w[1], v.w[2], v.w[3]};
  __builtin_nontemporal_store(x, static_cast<u32x4_any*>(p));
}

// Eight elements as they lie in memory, of which n exist (n >= 8: all; n <= 0: none).  load: one by one where n < 8.  load_end: where at least eight
// elements end at p + n, the eight that do; get_end moves them to their places, away from the load, which is then one instruction that nothing waits for.
template <class T> struct Raw8;
template <> struct Raw8<bf16_t> {
  Vec16 a{{0, 0, 0, 0}};
  __device__ __forceinline__ void load(const bf16_t* p, int n) {
    if (n >= 8) { a = load16(p); return; }
    a = Vec16{{0, 0, 0, 0}};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) a.w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
  }
  __device__ __forceinline__ void load_end(const bf16_t* p, int n) {
    if (n > 0) a = load16(p + (n < 8 ? n - 8 : 0));
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[2 * q] = __uint_as_float(a.w[q] << 16); v[2 * q + 1] = __uint_as_float(a.w[q] & 0xffff0000u); }
  }
};
template <> struct Raw8<float> {
  Vec16 a{{0, 0, 0, 0}}, b{{0, 0, 0, 0}};
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= 8) { a = load16(p); b = load16(p + 4); return; }
    a = b = Vec16{{0, 0, 0, 0}};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) (e < 4 ? a : b).w[e & 3] = __float_as_uint(p[e]);
  }
  __device__ __forceinline__ void load_end(const float* p, int n) {
    if (n > 0) {
      p += n < 8 ? n - 8 : 0;
      a = load16(p);
      b = load16(p + 4);
    }
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[q] = __uint_as_float(a.w[q]); v[4 + q] = __uint_as_float(b.w[q]); }
  }
};
template <class T>
__device__ __forceinline__ void get_end(const Raw8<T>& r, float* v, int n) {
  r.get(v);
  if (n < 8 && n > 0) {
    const int by = 8 - n;
#pragma unroll
    for (int step = 1; step < 8; step *= 2)
      if (by & step) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e + step < 8 ? v[e + step] : 0.f;
      }
  }
}
__device__ __forceinline__ void put8(bf16_t* p, const float* v, int n) {
  const Vec16 o{{f2bf_pair(v[0], v[1]), f2bf_pair(v[2], v[3]), f2bf_pair(v[4], v[5]), f2bf_pair(v[6], v[7])}};
  if (n >= 8) { store16(p, o); return; }
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) p[e] = (bf16_t)(o.w[e >> 1] >> (16 * (e & 1)));
}
__device__ __forceinline__ void put8(float* p, const float* v, int n) {
  if (n >= 8) {
    store16(p, Vec16{{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}});
    store16(p + 4, Vec16{{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}});
    return;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) p[e] = v[e];
}

// ---- clip.hip ----
size_t clip_work_bytes(const pbt_grad* g, int n, int P);
hipError_t clip_gradients(const pbt_grad* g, int n, int P, const float* max_norm, int64_t max_norm_stride, float* norm, void* work, hipStream_t s);

// The norm of G[P][stride] (all of it: padding is zero) and the factor that brings it down to max_norm[i * max_norm_stride]: norm[P], factor[P].
size_t grad_factor_work_bytes(int64_t stride, int P);
hipError_t grad_factor(const float* G, int64_t stride, int P, const float* max_norm, int64_t max_norm_stride, float* norm, float* factor, void* work, hipStream_t s);

// ---- rotary.hip ----
struct RotaryFrequencies { double turns[PBT_ROTARY_MAX_DIM / 2]; };
hipError_t rotary_plan(const RotaryFrequencies& f, int n, double* table, hipStream_t s);
// turns per position of every pair
void rotary_frequencies(const pbt_rotary& r, RotaryFrequencies* f);
// the same, refused where they are not finite (operators_abi.hip; settings that check_rotary lets pass)
pbt_status check_rotary_frequencies(const pbt_rotary* r, RotaryFrequencies* f);
struct RotaryArgs {
  pbt_heads g[4];
  int n_groups;
  int64_t rows;
  int width, rot;
  const void* pos;
  int pos64;
  int64_t start, period;
  float gain, sign;         // sign of the sine: -1 transposes
  const double* turns;
};
hipError_t rotary_apply(const RotaryArgs& a, int layout, int dtype, hipStream_t s);

// ---- block_norm_forward.hip, block_norm_backward.hip ----
struct BlockArgs {
  pbt_block_norm n;
  pbt_block_params p, g;    // parameters, their gradients
  pbt_rows y, x, gate, out, z, dout, dz, dy, dx, dgate;
  float* stats;
  float* part;
};
size_t block_norm_work_bytes(const pbt_block_norm& n);
hipError_t block_norm_forward(const BlockArgs& a, hipStream_t s);
hipError_t block_norm_backward(const BlockArgs& a, hipStream_t s);

}  // namespace pbt
