// How the operators' launches are cut up: rules on sizes alone.
#pragma once
#include <algorithm>
#include <cstdint>

namespace pbt {

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

}  // namespace pbt
