"""The operators' rules on sizes (csrc/operators_choose.h), compiled for the host, so that a test can say which kernel and cut its sizes reach."""
import collections
import ctypes
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1711_09846_amd", "csrc")
_SOURCE = r"""
#include "operators_choose.h"
extern "C" void rotary(int unit, int half, int rot, int width, long long rows, int n_groups, const int* heads, const int* apart, long long* out) {
  pbt::RotaryCall call{unit, half != 0, rot, width, rows, n_groups, {}, {}};
  for (int g = 0; g < n_groups; ++g) { call.heads[g] = heads[g]; call.apart[g] = apart[g] != 0; }
  const pbt::RotaryCut c = pbt::rotary_cut(call);
  *out++ = pbt::rotary_unit_pairs(unit, half != 0);
  *out++ = c.pitch; *out++ = c.table; *out++ = c.blocks;
  for (int g = 0; g < n_groups; ++g) {
    const pbt::RotaryShape& w = c.shapes.g[g];
    *out++ = w.rows; *out++ = w.heads; *out++ = w.head_blocks; *out++ = w.row_blocks; *out++ = w.pair_units; *out++ = w.units;
  }
}
"""


@functools.lru_cache(None)
def _lib():
    d = tempfile.mkdtemp()
    src, so = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
    with open(src, "w") as f:
        f.write(_SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
    return ctypes.CDLL(so)


RotaryGroup = collections.namedtuple("RotaryGroup", "rows heads head_blocks row_blocks pair_units units")
RotaryCut = collections.namedtuple("RotaryCut", "unit_pairs pitch table blocks groups")


def rotary(dtype, layout, rot, width, rows, heads, apart):
    """The cut of a rotary call: dtype "fp32" or "bf16", heads and apart (results go elsewhere) of its groups."""
    n = len(heads)
    out = (ctypes.c_longlong * (4 + 6 * n))()
    _lib().rotary(8 if dtype == "bf16" else 4, int(layout == "half"), rot, width, ctypes.c_longlong(rows), n, (ctypes.c_int * n)(*heads),
                  (ctypes.c_int * n)(*map(int, apart)), out)
    return RotaryCut(*out[:4], [RotaryGroup(*out[4 + 6 * g:10 + 6 * g]) for g in range(n)])
