// C ABI of the operators that need no handle: arguments are checked here, on the host, before anything is launched.
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <utility>

#include "handle.h"
#include "operators.h"
#include "operators_apart.h"

using namespace pbt;

namespace pbt {
pbt_status check_rotary(const pbt_rotary* r) {
  if (!r) return fail(nullptr, PBT_EINVAL, "rotary settings are NULL");
  if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > PBT_ROTARY_MAX_DIM) return fail(nullptr, PBT_EINVAL, "rot_dim = %d: even, 2..%d", r->rot_dim, PBT_ROTARY_MAX_DIM);
  if (r->layout != PBT_ROTARY_HALF && r->layout != PBT_ROTARY_INTERLEAVED) return fail(nullptr, PBT_EINVAL, "unknown rotary layout %d", r->layout);
  if (r->scaling < PBT_ROTARY_SCALE_NONE || r->scaling > PBT_ROTARY_SCALE_RAMP) return fail(nullptr, PBT_EINVAL, "unknown rotary scaling %d", r->scaling);
  if (r->unused != 0) return fail(nullptr, PBT_EINVAL, "the unused field must be 0");
  if (!(r->base > 0.0) || !std::isfinite(r->base)) return fail(nullptr, PBT_EINVAL, "base must be positive and finite");
  if (!std::isfinite((float)r->gain)) return fail(nullptr, PBT_EINVAL, "gain must be finite, as a float too");
  if (r->scaling != PBT_ROTARY_SCALE_NONE && (!(r->factor > 0.0) || !std::isfinite(r->factor))) return fail(nullptr, PBT_EINVAL, "factor must be positive and finite");
  if (r->scaling == PBT_ROTARY_SCALE_RAMP &&
      (!(r->trained_len > 0.0) || !std::isfinite(r->trained_len) || !(r->low < r->high) || !std::isfinite(r->low) || !std::isfinite(r->high)))
    return fail(nullptr, PBT_EINVAL, "ramp scaling needs trained_len > 0 and low < high, finite");
  return PBT_OK;
}
pbt_status check_rotary_frequencies(const pbt_rotary* r, RotaryFrequencies* f) {
  rotary_frequencies(*r, f);
  for (int j = 0; j < r->rot_dim / 2; ++j)
    if (!std::isfinite(f->turns[j])) return fail(nullptr, PBT_EINVAL, "base and factor take the frequency of pair %d out of range", j);
  return PBT_OK;
}
}  // namespace pbt

namespace {

size_t elem_bytes(int dtype) { return dtype == PBT_DTYPE_BF16 ? 2 : 4; }
bool known_dtype(int dtype) { return dtype == PBT_DTYPE_FP32 || dtype == PBT_DTYPE_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// [a, a + a_bytes) and [b, b + b_bytes) share a byte
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

constexpr int64_t MOST = (int64_t)1 << 46;   // lengths, strides and counts beyond it are mistakes (their products stay within 63 bits below)

pbt_status check_grads(const pbt_grad* g, int n, int P, bool clip) {
  if (!g || n < 1) return fail(nullptr, PBT_EINVAL, "no tensors are given");
  if (P < 1 || P > PBT_MAX_P) return fail(nullptr, PBT_EINVAL, "P = %d outside 1..%d", P, PBT_MAX_P);
  for (int k = 0; k < n; ++k) {
    const pbt_grad& t = g[k];
    if (!known_dtype(t.dtype)) return fail(nullptr, PBT_EINVAL, "tensor %d: unknown dtype %d", k, t.dtype);
    if (t.unused != 0) return fail(nullptr, PBT_EINVAL, "tensor %d: the unused field must be 0", k);
    if (t.len < 0 || t.len > MOST) return fail(nullptr, PBT_EINVAL, "tensor %d: length %lld outside 0..2^46", k, (long long)t.len);
    if (t.len == 0) continue;
    const size_t e = elem_bytes(t.dtype);
    if (!t.d_src || !aligned(t.d_src, e)) return fail(nullptr, PBT_EINVAL, "tensor %d: src is NULL or not aligned to its elements", k);
    if (P > 1 && (t.src_stride < t.len || t.src_stride > MOST)) return fail(nullptr, PBT_EINVAL, "tensor %d: src_stride below the length or above 2^46", k);
    if (!clip) continue;
    if (!t.d_dst || !aligned(t.d_dst, e)) return fail(nullptr, PBT_EINVAL, "tensor %d: dst is NULL or not aligned to its elements", k);
    if (P > 1 && (t.dst_stride < t.len || t.dst_stride > MOST)) return fail(nullptr, PBT_EINVAL, "tensor %d: dst_stride below the length or above 2^46", k);
    if (t.d_src == t.d_dst) {
      if (P > 1 && t.src_stride != t.dst_stride) return fail(nullptr, PBT_EINVAL, "tensor %d: clipped in place with two strides", k);
    } else {
      const int64_t a = ((P - 1) * t.src_stride + t.len) * (int64_t)e, b = ((P - 1) * t.dst_stride + t.len) * (int64_t)e;
      if (overlap(t.d_src, a, t.d_dst, b)) {
        // rows of one array side by side are fine
        const int64_t diff = static_cast<const char*>(t.d_dst) - static_cast<const char*>(t.d_src);
        const int64_t p = t.src_stride * (int64_t)e;
        const int64_t m = P > 1 && t.src_stride == t.dst_stride ? ((diff % p) + p) % p : 0;
        if (m < t.len * (int64_t)e || p - m < t.len * (int64_t)e) return fail(nullptr, PBT_EINVAL, "tensor %d: src and dst overlap", k);
      }
    }
  }
  return PBT_OK;
}

// What a call writes is apart from everything else that it touches (a tensor's own src and dst have been looked at).  max_norm NULL: norms only, no dst is written.
pbt_status check_grads_apart(const pbt_grad* g, int n, int P, const float* max_norm, int64_t max_norm_stride, float* norm, void* work, size_t work_bytes) {
  constexpr int FEW = 256;
  Region few[FEW], *r = few;
  RegionKey few_keys[FEW], *keys = few_keys;
  std::unique_ptr<Region[]> many;
  std::unique_ptr<RegionKey[]> many_keys;
  const size_t most = 2 * (size_t)n + 3;
  if (most > FEW) {
    many.reset(new (std::nothrow) Region[most]);
    many_keys.reset(new (std::nothrow) RegionKey[most]);
    r = many.get();
    keys = many_keys.get();
    if (!r || !keys) return fail(nullptr, PBT_ENOMEM, "out of host memory");
  }
  enum { NORM = -1, MAX_NORM = -2, WORK = -3 };
  int m = 0;
  for (int k = 0; k < n; ++k) {
    if (g[k].len == 0) continue;
    const int64_t e = (int64_t)elem_bytes(g[k].dtype);
    if (max_norm) r[m++] = Region{reinterpret_cast<uintptr_t>(g[k].d_dst), g[k].len * e, P > 1 ? g[k].dst_stride * e : 0, P, true, k};
    if (!max_norm || g[k].d_src != g[k].d_dst) r[m++] = Region{reinterpret_cast<uintptr_t>(g[k].d_src), g[k].len * e, P > 1 ? g[k].src_stride * e : 0, P, false, k};
  }
  if (max_norm) r[m++] = Region{reinterpret_cast<uintptr_t>(max_norm), 4, max_norm_stride * 4, max_norm_stride > 0 ? P : 1, false, MAX_NORM};
  if (norm) r[m++] = Region{reinterpret_cast<uintptr_t>(norm), (int64_t)P * 4, 0, 1, true, NORM};
  r[m++] = Region{reinterpret_cast<uintptr_t>(work), (int64_t)work_bytes, 0, 1, true, WORK};
  int x, y;
  if (!find_meeting(r, keys, m, &x, &y)) return PBT_OK;
  if (x > y) std::swap(x, y);
  if (x >= 0) return fail(nullptr, PBT_EINVAL, "dst of one of the tensors %d and %d overlaps the other", x, y);
  const char* const names[3] = {"norm", "max_norm", "the working memory"};
  if (y >= 0) return fail(nullptr, PBT_EINVAL, "%s overlaps tensor %d", names[-1 - x], y);
  return fail(nullptr, PBT_EINVAL, "%s overlaps %s", names[-1 - x], names[-1 - y]);
}

HeadView src_view(const pbt_heads& g, int64_t rows, int width, int64_t e) {
  return HeadView{reinterpret_cast<uintptr_t>(g.d_src), g.src_row * e, g.src_head * e, rows, g.heads, width * e};
}
HeadView dst_view(const pbt_heads& g, int64_t rows, int width, int64_t e) {
  return HeadView{reinterpret_cast<uintptr_t>(g.d_dst), g.dst_row * e, g.dst_head * e, rows, g.heads, width * e};
}
bool same_view(const pbt_heads& g, int64_t rows) {
  return g.d_src == g.d_dst && (rows == 1 || g.src_row == g.dst_row) && (g.heads == 1 || g.src_head == g.dst_head);
}

pbt_status check_block(const pbt_block_norm* n) {
  if (!n) return fail(nullptr, PBT_EINVAL, "block norm settings are NULL");
  if (n->P < 1 || n->P > PBT_MAX_P) return fail(nullptr, PBT_EINVAL, "P = %d outside 1..%d", n->P, PBT_MAX_P);
  if (n->rows < 0 || n->rows > ((int64_t)1 << 40)) return fail(nullptr, PBT_EINVAL, "rows outside 0..2^40");
  if (n->d < 1) return fail(nullptr, PBT_EINVAL, "d must be positive");
  if (n->d > PBT_BLOCK_NORM_MAX_D) return fail(nullptr, PBT_EUNSUPPORTED, "d = %d: rows of up to %d elements are built", n->d, PBT_BLOCK_NORM_MAX_D);
  if (n->post < PBT_NORM_NONE || n->post > PBT_NORM_RMS || n->pre < PBT_NORM_NONE || n->pre > PBT_NORM_RMS) return fail(nullptr, PBT_EINVAL, "unknown norm %d / %d", n->post, n->pre);
  if (n->post == PBT_NORM_NONE && n->pre == PBT_NORM_NONE) return fail(nullptr, PBT_EINVAL, "neither a norm after the block nor one before the next");
  if (n->gate < PBT_GATE_NONE || n->gate > PBT_GATE_ROWS) return fail(nullptr, PBT_EINVAL, "unknown gate %d", n->gate);
  if (n->gate_act != PBT_ACT_NONE && n->gate_act != PBT_ACT_SIGMOID && n->gate_act != PBT_ACT_SILU && n->gate_act != PBT_ACT_TANH)
    return fail(nullptr, PBT_EINVAL, "activation %d is none of a gate's", n->gate_act);
  if (n->gate == PBT_GATE_NONE && n->gate_act != PBT_ACT_NONE) return fail(nullptr, PBT_EINVAL, "a gate activation without a gate");
  if (!known_dtype(n->dtype) || !known_dtype(n->res_dtype)) return fail(nullptr, PBT_EINVAL, "unknown dtype %d / %d", n->dtype, n->res_dtype);
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps) || !std::isfinite(n->alpha) || !std::isfinite(n->beta)) return fail(nullptr, PBT_EINVAL, "eps >= 0, alpha and beta must be finite");
  return PBT_OK;
}

// a matrix of a block norm: there (unless optional), aligned to its elements, rows that do not overlap
pbt_status check_rows(const pbt_block_norm* n, const pbt_rows* m, const char* name, int dtype, bool optional) {
  if (!m || !m->d) return optional ? PBT_OK : fail(nullptr, PBT_EINVAL, "%s is NULL", name);
  if (!aligned(m->d, elem_bytes(dtype))) return fail(nullptr, PBT_EINVAL, "%s is not aligned to its elements", name);
  if (m->pitch < n->d || m->pitch > ((int64_t)1 << 32)) return fail(nullptr, PBT_EINVAL, "%s: pitch %lld below d or above 2^32", name, (long long)m->pitch);
  if ((int64_t)n->P * n->rows > MOST / m->pitch) return fail(nullptr, PBT_EINVAL, "%s is too large", name);
  return PBT_OK;
}
pbt_status check_params(const pbt_block_norm* n, const pbt_block_params* p, const char* what) {
  if (!p) return fail(nullptr, PBT_EINVAL, "%s are NULL", what);
  float* const* q = &p->post_gain;
  for (int k = 0; k < 5; ++k)
    if (q[k] && !aligned(q[k], 4)) return fail(nullptr, PBT_EINVAL, "%s: pointer %d is not aligned to its elements", what, k);
  if (n->P > 1 && (q[0] || q[1] || q[2] || q[3] || q[4]) && (p->stride < n->d || p->stride > MOST)) return fail(nullptr, PBT_EINVAL, "%s: stride below d or above 2^46", what);
  return PBT_OK;
}
// What a block norm's call reads and writes, by name.
struct BlockMemory {
  const pbt_block_norm* n;
  Region r[24];
  const char* names[24];
  int count = 0;
  void add(const void* p, int64_t bytes, int64_t stride, int64_t pieces, bool written, const char* name) {
    if (!p) return;
    names[count] = name;
    r[count] = Region{reinterpret_cast<uintptr_t>(p), bytes, stride, pieces, written, count};
    ++count;
  }
  void add_rows(const pbt_rows* m, int type, bool written, const char* name) {
    if (!m || !m->d || n->rows == 0) return;
    const int64_t e = (int64_t)elem_bytes(type), rows = n->P * n->rows;
    if (m->pitch == n->d) add(m->d, rows * n->d * e, 0, 1, written, name);
    else add(m->d, n->d * e, m->pitch * e, rows, written, name);
  }
  // an input that an output may lie over: looked at where that is not the same rows
  void add_rows_apart_from(const pbt_rows* m, int type, const char* name, const pbt_rows& out) {
    if (m && m->d == out.d && m->pitch == out.pitch) return;
    add_rows(m, type, false, name);
  }
  // (one member's stride is not looked at, and may be anything)
  void add_params(const pbt_block_params* p, bool written, const char* const* name) {
    float* const* q = &p->post_gain;
    for (int k = 0; k < 5; ++k) add(q[k], (int64_t)n->d * 4, n->P > 1 ? p->stride * 4 : 0, n->P, written, name[k]);
  }
  pbt_status check() {
    RegionKey keys[24];
    int x, y;
    if (!find_meeting(r, keys, count, &x, &y)) return PBT_OK;
    return fail(nullptr, PBT_EINVAL, "%s overlaps %s", names[x], names[y]);
  }
};
const char* const PARAM_NAMES[5] = {"post_gain", "post_bias", "pre_gain", "pre_bias", "the gate vector"};
const char* const GRAD_NAMES[5] = {"the gradient of post_gain", "the gradient of post_bias", "the gradient of pre_gain", "the gradient of pre_bias", "the gate vector's gradient"};

#define TRY(call) do { const pbt_status st_ = (call); if (st_ != PBT_OK) return st_; } while (0)

}  // namespace

extern "C" {

pbt_status pbt_clip_work_bytes(const pbt_grad* h_grads, int32_t n_grads, int32_t P, size_t* bytes) {
  if (!bytes) return fail(nullptr, PBT_EINVAL, "bytes is NULL");
  TRY(check_grads(h_grads, n_grads, P, false));
  *bytes = clip_work_bytes(h_grads, n_grads, P);
  return PBT_OK;
}

pbt_status pbt_clip_gradients(const pbt_grad* h_grads, int32_t n_grads, int32_t P, const float* d_max_norm, int64_t max_norm_stride, float* d_norm, void* d_work,
                              size_t work_bytes, void* hip_stream) {
  TRY(check_grads(h_grads, n_grads, P, d_max_norm != nullptr));
  if (!aligned(d_max_norm, 4) || !aligned(d_norm, 4)) return fail(nullptr, PBT_EINVAL, "max_norm and norm must be aligned to floats");
  if (d_max_norm && (max_norm_stride < 0 || max_norm_stride > MOST)) return fail(nullptr, PBT_EINVAL, "max_norm_stride outside 0..2^46");
  if (!d_max_norm && !d_norm) return fail(nullptr, PBT_EINVAL, "neither a bound nor a place for the norms");
  const size_t need = clip_work_bytes(h_grads, n_grads, P);
  if (!d_work || !aligned(d_work, 8)) return fail(nullptr, PBT_EINVAL, "work is NULL or not 8-byte aligned");
  if (work_bytes < need) return fail(nullptr, PBT_ENOMEM, "working memory: %zu bytes given, %zu needed", work_bytes, need);
  TRY(check_grads_apart(h_grads, n_grads, P, d_max_norm, max_norm_stride, d_norm, d_work, need));
  const hipError_t e = clip_gradients(h_grads, n_grads, P, d_max_norm, max_norm_stride, d_norm, d_work, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail(nullptr, PBT_EDEVICE, "clipping failed to launch: %s", hipGetErrorString(e));
  return PBT_OK;
}

pbt_status pbt_rotary_plan(const pbt_rotary* r, void* d_table, size_t table_bytes, void* hip_stream) {
  TRY(check_rotary(r));
  if (!d_table || !aligned(d_table, 8)) return fail(nullptr, PBT_EINVAL, "table is NULL or not 8-byte aligned");
  const int pairs = r->rot_dim / 2;
  if (table_bytes < pairs * sizeof(double)) return fail(nullptr, PBT_ENOMEM, "table: %zu bytes given, %zu needed", table_bytes, pairs * sizeof(double));
  RotaryFrequencies f;
  TRY(check_rotary_frequencies(r, &f));
  const hipError_t e = rotary_plan(f, pairs, static_cast<double*>(d_table), static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail(nullptr, PBT_EDEVICE, "writing the rotary table failed: %s", hipGetErrorString(e));
  return PBT_OK;
}

pbt_status pbt_rotary_apply(const pbt_rotary* r, const void* d_table, const pbt_heads* h_groups, int32_t n_groups, int32_t dtype, int64_t rows, int32_t width,
                            const void* d_positions, int32_t position_bytes, int64_t start, int64_t period, int32_t backward, void* hip_stream) {
  TRY(check_rotary(r));
  if (!d_table || !aligned(d_table, 8)) return fail(nullptr, PBT_EINVAL, "table is NULL or not 8-byte aligned");
  if (!h_groups || n_groups < 1 || n_groups > 4) return fail(nullptr, PBT_EINVAL, "1 to 4 groups of heads");
  if (!known_dtype(dtype)) return fail(nullptr, PBT_EINVAL, "unknown dtype %d", dtype);
  if (rows < 0 || rows > 0x7fffffffLL) return fail(nullptr, PBT_EINVAL, "rows outside 0..2^31-1");
  if (width < r->rot_dim || width > 16384) return fail(nullptr, PBT_EINVAL, "heads of %d elements: rot_dim (%d) to 16384", width, r->rot_dim);
  if (d_positions && position_bytes != 4 && position_bytes != 8) return fail(nullptr, PBT_EINVAL, "positions have 4 or 8 bytes");
  if (d_positions && !aligned(d_positions, position_bytes)) return fail(nullptr, PBT_EINVAL, "positions are not aligned to their elements");
  if (!d_positions && (period < 0 || start < -MOST || start > MOST)) return fail(nullptr, PBT_EINVAL, "period below 0, or start outside +-2^46");
  if (backward != 0 && backward != 1) return fail(nullptr, PBT_EINVAL, "backward is 0 or 1");
  const int64_t e = (int64_t)elem_bytes(dtype);
  int64_t heads = 0;
  for (int k = 0; k < n_groups; ++k) {
    const pbt_heads& g = h_groups[k];
    if (g.heads < 1 || g.heads > 32768) return fail(nullptr, PBT_EINVAL, "group %d: heads outside 1..32768", k);
    if (g.unused != 0) return fail(nullptr, PBT_EINVAL, "group %d: the unused field must be 0", k);
    heads += g.heads;
    if (rows == 0) continue;
    if (!g.d_src || !g.d_dst || !aligned(g.d_src, e) || !aligned(g.d_dst, e)) return fail(nullptr, PBT_EINVAL, "group %d: src or dst is NULL or not aligned to its elements", k);
    if (g.heads > 1 && (g.src_head < width || g.dst_head < width)) return fail(nullptr, PBT_EINVAL, "group %d: heads overlap", k);
    const int64_t limit = (int64_t)1 << 31;
    if (g.src_row < 0 || g.dst_row < 0 || g.src_head > limit || g.dst_head > limit || g.src_row > limit || g.dst_row > limit)
      return fail(nullptr, PBT_EINVAL, "group %d: strides above 2^31 or negative", k);
    if (rows > 1 && std::max(g.src_row, g.dst_row) > MOST / (rows - 1)) return fail(nullptr, PBT_EINVAL, "group %d: rows span more than 2^46 elements", k);
    // dst's elements are apart: heads within rows, or rows within heads
    const bool in_rows = g.dst_row >= (g.heads - 1) * g.dst_head + width, in_heads = g.dst_row >= width && g.dst_head >= (rows - 1) * g.dst_row + width;
    if (rows > 1 && !(g.heads == 1 ? g.dst_row >= width : in_rows || in_heads)) return fail(nullptr, PBT_EINVAL, "group %d: rows of dst overlap", k);
    if (!same_view(g, rows) && !heads_apart(src_view(g, rows, width, e), dst_view(g, rows, width, e))) return fail(nullptr, PBT_EINVAL, "group %d: dst overlaps src and is not the same view", k);
  }
  for (int k = 0; k < n_groups && rows > 0; ++k)
    for (int j = 0; j < n_groups; ++j) {
      if (j == k) continue;
      const HeadView out = dst_view(h_groups[k], rows, width, e);
      if (!heads_apart(out, src_view(h_groups[j], rows, width, e)) || !heads_apart(out, dst_view(h_groups[j], rows, width, e)))
        return fail(nullptr, PBT_EINVAL, "dst of group %d overlaps group %d", k, j);
    }
  for (int k = 0; k < n_groups && rows > 0; ++k) {
    const HeadView out = dst_view(h_groups[k], rows, width, e);
    const auto under = [&](const void* p, int64_t bytes) { return p && !heads_apart(out, HeadView{reinterpret_cast<uintptr_t>(p), out.row, 0, 1, 1, bytes}); };
    if (under(d_positions, rows * position_bytes)) return fail(nullptr, PBT_EINVAL, "dst of group %d overlaps the positions", k);
    if (under(d_table, r->rot_dim / 2 * 8)) return fail(nullptr, PBT_EINVAL, "dst of group %d overlaps the table", k);
  }
  if (heads > 32768) return fail(nullptr, PBT_EINVAL, "more than 32768 heads");
  if (rows == 0) return PBT_OK;
  RotaryArgs a;
  std::memset(&a, 0, sizeof a);
  for (int k = 0; k < n_groups; ++k) a.g[k] = h_groups[k];
  a.n_groups = n_groups;
  a.rows = rows; a.width = width; a.rot = r->rot_dim;
  a.pos = d_positions; a.pos64 = position_bytes == 8;
  a.start = start; a.period = period;
  a.gain = (float)r->gain; a.sign = backward ? -1.f : 1.f;
  a.turns = static_cast<const double*>(d_table);
  const hipError_t err = rotary_apply(a, r->layout, dtype, static_cast<hipStream_t>(hip_stream));
  if (err != hipSuccess) return fail(nullptr, PBT_EDEVICE, "rotary positions failed to launch: %s", hipGetErrorString(err));
  return PBT_OK;
}

pbt_status pbt_block_norm_forward(const pbt_block_norm* n, const pbt_rows* y, const pbt_rows* x, const pbt_rows* gate, const pbt_block_params* params,
                                  const pbt_rows* out, const pbt_rows* z, float* d_stats, void* hip_stream) {
  TRY(check_block(n));
  const int A = n->dtype, R = n->res_dtype;
  const bool gated = n->gate == PBT_GATE_ROWS, normed = n->pre != PBT_NORM_NONE;
  TRY(check_params(n, params, "parameters"));
  if (n->gate == PBT_GATE_VECTOR && !params->gate) return fail(nullptr, PBT_EINVAL, "the gate vector is NULL");
  if (n->rows == 0) return PBT_OK;
  TRY(check_rows(n, y, "y", A, false));
  TRY(check_rows(n, x, "x", R, false));
  if (gated) TRY(check_rows(n, gate, "gate", A, false));
  TRY(check_rows(n, out, "out", R, false));
  if (normed) TRY(check_rows(n, z, "z", A, false));
  if (!aligned(d_stats, 16)) return fail(nullptr, PBT_EINVAL, "stats must be 16-byte aligned");
  BlockMemory memory{n};
  memory.add_rows(out, R, true, "out");
  memory.add_rows_apart_from(x, R, "x", *out);
  if (normed) {
    memory.add_rows(z, A, true, "z");
    memory.add_rows_apart_from(y, A, "y", *z);
  } else {
    memory.add_rows(y, A, false, "y");
  }
  if (gated) memory.add_rows(gate, A, false, "the gate");
  memory.add(d_stats, n->P * n->rows * 16, 0, 1, true, "stats");
  memory.add_params(params, false, PARAM_NAMES);
  TRY(memory.check());
  BlockArgs a;
  std::memset(&a, 0, sizeof a);
  a.n = *n; a.p = *params; a.y = *y; a.x = *x; a.out = *out; a.stats = d_stats;
  if (gated) a.gate = *gate;
  if (normed) a.z = *z;
  const hipError_t e = block_norm_forward(a, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail(nullptr, PBT_EDEVICE, "block norm failed to launch: %s", hipGetErrorString(e));
  return PBT_OK;
}

pbt_status pbt_block_norm_work_bytes(const pbt_block_norm* n, size_t* bytes) {
  if (!bytes) return fail(nullptr, PBT_EINVAL, "bytes is NULL");
  TRY(check_block(n));
  *bytes = block_norm_work_bytes(*n);
  return PBT_OK;
}

pbt_status pbt_block_norm_backward(const pbt_block_norm* n, const pbt_rows* y, const pbt_rows* x, const pbt_rows* gate, const pbt_block_params* params,
                                   const float* d_stats, const pbt_rows* dout, const pbt_rows* dz, const pbt_rows* dy, const pbt_rows* dx, const pbt_rows* dgate,
                                   const pbt_block_params* grads, void* d_work, size_t work_bytes, void* hip_stream) {
  TRY(check_block(n));
  const int A = n->dtype, R = n->res_dtype;
  const bool gated = n->gate == PBT_GATE_ROWS, normed = n->pre != PBT_NORM_NONE;
  TRY(check_params(n, params, "parameters"));
  TRY(check_params(n, grads, "parameter gradients"));
  if (n->gate == PBT_GATE_VECTOR && !params->gate) return fail(nullptr, PBT_EINVAL, "the gate vector is NULL");
  if (n->gate != PBT_GATE_VECTOR && grads->gate) return fail(nullptr, PBT_EINVAL, "a gradient of the gate vector is asked for and there is none");
  if (n->post == PBT_NORM_NONE && (grads->post_gain || grads->post_bias)) return fail(nullptr, PBT_EINVAL, "gradients of a norm after the block are asked for and there is none");
  if (!normed && (grads->pre_gain || grads->pre_bias)) return fail(nullptr, PBT_EINVAL, "gradients of a norm before the next block are asked for and there is none");
  const bool has_dz = normed && dz && dz->d, has_dout = dout && dout->d;
  if (n->rows > 0) {
    TRY(check_rows(n, y, "y", A, false));
    TRY(check_rows(n, x, "x", R, false));
    if (gated) TRY(check_rows(n, gate, "gate", A, false));
    if (gated) TRY(check_rows(n, dgate, "dgate", A, false));
    if (!has_dz && !has_dout) return fail(nullptr, PBT_EINVAL, "neither dout nor dz");
    if (has_dz) TRY(check_rows(n, dz, "dz", A, false));
    if (has_dout) TRY(check_rows(n, dout, "dout", R, false));
    TRY(check_rows(n, dy, "dy", A, false));
    TRY(check_rows(n, dx, "dx", R, false));
    if (!d_stats || !aligned(d_stats, 16)) return fail(nullptr, PBT_EINVAL, "stats is NULL or not 16-byte aligned");
    const size_t need = block_norm_work_bytes(*n);
    if (!d_work || !aligned(d_work, 16)) return fail(nullptr, PBT_EINVAL, "work is NULL or not 16-byte aligned");
    if (work_bytes < need) return fail(nullptr, PBT_ENOMEM, "working memory: %zu bytes given, %zu needed", work_bytes, need);
  }
  BlockMemory memory{n};
  if (n->rows > 0) {
    memory.add_rows(dy, A, true, "dy");
    memory.add_rows(dx, R, true, "dx");
    memory.add_rows(y, A, false, "y");
    memory.add_rows(x, R, false, "x");
    if (has_dz) memory.add_rows_apart_from(dz, A, "dz", *dy);
    if (has_dout) memory.add_rows_apart_from(dout, R, "dout", *dx);
    if (gated) {
      memory.add_rows(dgate, A, true, "dgate");
      memory.add_rows(gate, A, false, "the gate");
    }
    memory.add(d_stats, n->P * n->rows * 16, 0, 1, false, "stats");
    memory.add(d_work, (int64_t)block_norm_work_bytes(*n), 0, 1, true, "the working memory");
  }
  memory.add_params(params, false, PARAM_NAMES);
  memory.add_params(grads, true, GRAD_NAMES);
  TRY(memory.check());
  BlockArgs a;
  std::memset(&a, 0, sizeof a);
  a.n = *n; a.p = *params; a.g = *grads;
  a.stats = const_cast<float*>(d_stats);
  a.part = static_cast<float*>(d_work);
  if (n->rows > 0) {
    a.y = *y; a.x = *x; a.dy = *dy; a.dx = *dx;
    if (gated) { a.gate = *gate; a.dgate = *dgate; }
    if (has_dz) a.dz = *dz;
    if (has_dout) a.dout = *dout;
  }
  const hipError_t e = block_norm_backward(a, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail(nullptr, PBT_EDEVICE, "block norm backward failed to launch: %s", hipGetErrorString(e));
  return PBT_OK;
}

}  // extern "C"
