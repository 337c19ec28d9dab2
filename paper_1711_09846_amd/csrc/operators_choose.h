// How the operators' launches are cut up: rules on sizes alone.
#pragma once
#include <algorithm>
#include <cstdint>

#include "../../include/pbt.h"

namespace pbt {

constexpr int64_t LAST_CACHE = (int64_t)256 << 20;   // bytes of the cache in front of memory: what a call writes beyond it is not found there afterwards

// ---- clip.hip ----
constexpr int CLIP_TENSORS = 64;          // of one launch (the table is a kernel argument)
constexpr int CLIP_HELD_THREADS = 1024;
inline int64_t clip_units(const pbt_grad& g) { return (g.len + 7) / 8; }
inline int64_t clip_units_of(const pbt_grad* g, int k0, int n) {
  int64_t total = 0;
  for (int k = k0; k < n && k < k0 + CLIP_TENSORS; ++k) total += clip_units(g[k]);
  return total;
}
// Units a thread holds where members are held, 0: they are not.  A workgroup a member: up to 4 units a thread whatever the number of members (one of 30000 floats:
// 5 us, 7 in two launches), 8 where there are members for a quarter of the compute units (128 of 60000 floats: 16 us, 20 in two launches; one: 10.5, 7.0).
inline int clip_held(const pbt_grad* g, int n, int P) {
  if (n > CLIP_TENSORS) return 0;
  const int64_t u = clip_units_of(g, 0, n);
  return u <= 4 * CLIP_HELD_THREADS ? 4 : u <= 8 * CLIP_HELD_THREADS && P >= 64 ? 8 : 0;
}
// ranges of a launch over `total` units of each of P members: at least `least` units each, about `grid` workgroups, at most `most` a member
inline int64_t clip_ranges_of(int64_t total, int P, int64_t least, int64_t grid, int64_t most) {
  return std::max<int64_t>(std::min(std::min((total + least - 1) / least, most), std::max<int64_t>(grid / P, 1)), 1);
}
// (Sums: a member's few hundred ranges are added up again by every workgroup of the second launch.  8192 workgroups instead of 2048: 128 x 202k floats 62 us
// instead of 60.  Factors: 16 x 21M floats take 762 us with 8192 workgroups, 743 with 32768.)
inline int64_t clip_sum_ranges(int64_t total, int P) { return clip_ranges_of(total, P, 256, 2048, 1024); }
inline int64_t clip_scale_ranges(int64_t total, int P) { return clip_ranges_of(total, P, 1024, 32768, 32768); }
inline int64_t clip_parts(const pbt_grad* g, int n, int P) {
  int64_t sum = 0;
  for (int k0 = 0; k0 < n; k0 += CLIP_TENSORS) sum += clip_sum_ranges(clip_units_of(g, k0, n), P);
  return sum;
}
// The products of a large call go past the caches.  (128 x 202k floats, 104 MB: 63 us so, 72 through the caches; 37 MB: no difference)
inline bool clip_past_caches(int64_t bytes) { return bytes > LAST_CACHE / 4; }

// ---- rotary.hip ----
struct RotaryShape {             // of a group of heads
  int64_t blocks;                // workgroups
  int rows, heads;               // of a workgroup
  int head_blocks, row_blocks;   // blocks = head_blocks row_blocks
  int pair_units, units;         // of a head: units of pairs, then those of the part that is copied
  uint32_t by_units, by_heads, by_pitch;
};
struct RotaryShapes { RotaryShape g[4]; };
struct RotaryCall {
  int unit;                      // elements of a 16-byte unit
  bool half;                     // layout: a pair's halves lie apart
  int rot, width;
  int64_t rows;
  int n_groups, heads[4];
  bool apart[4];                 // results go elsewhere
};
struct RotaryCut {
  RotaryShapes shapes;
  int pitch;                     // floats between a row's cosines and the next row's
  int table;                     // floats of LDS: [rows][pitch] cosines, then sines
  int64_t blocks;
};
// pairs of a unit
constexpr int rotary_unit_pairs(int unit, bool half) { return half ? unit : unit / 2; }
// A unit that is not whole reads the angles of a whole one, so a row of the table ends with one.
inline int rotary_pitch(int pairs, int unit_pairs) {
  const int to = std::max(unit_pairs, 4);
  return (pairs + to - 1) / to * to;
}
inline uint32_t rotary_magic(int d) { return d <= 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }   // (see quotient)

inline RotaryCut rotary_cut(const RotaryCall& a) {
  const int V = a.unit, PV = rotary_unit_pairs(V, a.half), pairs = a.rot / 2, pitch = rotary_pitch(pairs, PV);
  RotaryCut cut{};
  cut.pitch = pitch;
  int most_rows = 1;
  for (int g = 0; g < a.n_groups; ++g) {
    RotaryShape& w = cut.shapes.g[g];
    w.pair_units = (pairs + PV - 1) / PV;
    w.units = w.pair_units + (a.apart[g] ? (a.width - a.rot + V - 1) / V : 0);
    w.heads = std::min(std::max(2048 / w.units, 1), a.heads[g]);
    w.head_blocks = (a.heads[g] + w.heads - 1) / w.heads;
    // A table in LDS serves few rows: the first number of them whose units fill nine tenths of the workgroup's last sweep (else the one that does best), while
    // four workgroups are left for every compute unit and the table takes at most 16 KB.
    const int per_row = w.heads * w.units;
    const int64_t limit = std::min<int64_t>(std::min<int64_t>(2048 / pitch, 2048 / per_row + 1), a.rows * w.head_blocks / 1024);
    int64_t rows = 1;
    double best = 0.0;
    for (int64_t r = 1; r <= std::max<int64_t>(limit, 1) && best < 0.9; ++r) {
      const int64_t n = r * per_row;
      const double used = (double)n / (double)((n + 255) / 256 * 256);
      if (used > best) {
        best = used;
        rows = r;
      }
    }
    w.rows = (int)rows;
    w.by_units = rotary_magic(w.units);
    w.by_heads = rotary_magic(w.heads);
    w.by_pitch = rotary_magic(pitch);
    // (a grid holds 2^32 threads: the workgroups of a group take several blocks of rows where there would be more than 2^21 of them)
    w.row_blocks = (int)std::min((a.rows + rows - 1) / rows, std::max<int64_t>((1 << 21) / w.head_blocks, 1));
    w.blocks = (int64_t)w.row_blocks * w.head_blocks;
    cut.blocks += w.blocks;
    most_rows = std::max(most_rows, w.rows);
  }
  cut.table = 2 * most_rows * pitch;
  return cut;
}
// (Passes replayed from a graph: 131072 rows, 1.3 GB: 494 us past the caches, 513 through them; 65536 rows, 134 MB: 63 and 58.)
inline bool rotary_past_caches(int64_t bytes) { return bytes > LAST_CACHE; }

// ---- block_norm_forward.hip, block_norm_backward.hip ----
constexpr int WIDE = 0;   // T of a team that is the whole workgroup
struct BlockTeam { int T, threads, rows; };   // threads of a workgroup, rows it has at a time
inline BlockTeam block_team(int d) {
  if (d <= 64) return {8, 256, 32};
  if (d <= 128) return {16, 256, 16};
  if (d <= 256) return {32, 256, 8};
  if (d <= 512) return {64, 256, 4};
  return {WIDE, (d + 511) / 512 * 64, 1};
}

// Rows of a slab.  What a slab costs besides its rows (`extra` bytes a column: parameters read, sums written and read again) should be an eighth of what
// its rows move (`moved` bytes a column and row) and a team should see eight rows, while every compute unit has `resident` workgroups, and there
// are at most `most` in all.
inline int64_t slab_rows(const pbt_block_norm& n, int extra, int moved, int resident, int most) {
  const BlockTeam t = block_team(n.d);
  const int64_t all = n.rows * n.P;
  int64_t rows = std::max<int64_t>((8 * extra + moved - 1) / moved, 8 * t.rows);
  rows = std::min(rows, (all + 256 * resident - 1) / (256 * resident));   // (rounded up: a few workgroups more than fit would double the time)
  rows = std::max(rows, (all + most - 1) / most);
  rows = (rows + t.rows - 1) / t.rows * t.rows;
  return std::max<int64_t>(std::min(rows, n.rows), 1);
}
inline int64_t block_forward_slab(const pbt_block_norm& n, int params) {
  const int a = n.dtype == PBT_DTYPE_BF16 ? 2 : 4, r = n.res_dtype == PBT_DTYPE_BF16 ? 2 : 4;
  const int moved = (n.pre != PBT_NORM_NONE ? 2 : 1) * a + (n.gate == PBT_GATE_ROWS ? a : 0) + 2 * r;
  return slab_rows(n, 4 * params, moved, std::max(16 / (block_team(n.d).threads / 64), 1), 4096);
}
// (every gradient counted: the working memory does not depend on which are asked for)
inline int64_t block_backward_slab(const pbt_block_norm& n) {
  const int a = n.dtype == PBT_DTYPE_BF16 ? 2 : 4, r = n.res_dtype == PBT_DTYPE_BF16 ? 2 : 4;
  const int norms = (n.post != PBT_NORM_NONE) + (n.pre != PBT_NORM_NONE), sums = 2 * norms + (n.gate == PBT_GATE_VECTOR);
  const int moved = (n.pre != PBT_NORM_NONE ? 3 : 2) * a + (n.gate == PBT_GATE_ROWS ? 2 * a : 0) + 3 * r;
  return slab_rows(n, 4 * sums + 8 * sums, moved, std::max(8 / (block_team(n.d).threads / 64), 1), 2048);
}
inline bool block_ends_alone(int d) { return d < 8 || (d > 512 && d % 512 > 0 && d % 512 < 8); }

}  // namespace pbt
