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
extern "C" void block(long long rows, int P, int d, int post, int pre, int gate, int dtype, int res, int params, long long* out) {
  const pbt_block_norm n{rows, P, d, post, pre, gate, 0, dtype, res, 1e-5f, 1.f, 1.f};
  const pbt::BlockTeam t = pbt::block_team(d);
  *out++ = t.T; *out++ = t.threads; *out++ = t.rows; *out++ = pbt::block_ends_alone(d);
  *out++ = pbt::block_forward_slab(n, params); *out++ = pbt::block_backward_slab(n);
}
extern "C" void clip(const long long* sizes, const int* dtypes, int n, int P, long long* out) {
  pbt_grad* g = new pbt_grad[n];
  long long bytes = 0;
  for (int k = 0; k < n; ++k) {
    g[k] = pbt_grad{nullptr, nullptr, sizes[k], sizes[k], sizes[k], dtypes[k], 0};
    bytes += P * sizes[k] * (dtypes[k] == PBT_DTYPE_BF16 ? 2 : 4);
  }
  *out++ = pbt::clip_held(g, n, P); *out++ = pbt::clip_past_caches(bytes); *out++ = pbt::clip_parts(g, n, P); *out++ = (n + pbt::CLIP_TENSORS - 1) / pbt::CLIP_TENSORS;
  delete[] g;
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


BlockCut = collections.namedtuple("BlockCut", "T threads team_rows alone forward backward")     # forward, backward: rows of a slab
_NORMS, _GATES, _TYPES = {"none": 0, "layer": 1, "rms": 2}, {"none": 0, "vector": 1, "rows": 2}, {"fp32": 0, "bf16": 1}


def block(P, rows, d, post, pre, gate, dtype, res, params):
    """The cut of a block norm's passes; params: how many parameters the forward pass is given."""
    out = (ctypes.c_longlong * 6)()
    _lib().block(ctypes.c_longlong(rows), P, d, _NORMS[post], _NORMS[pre], _GATES[gate], _TYPES[dtype], _TYPES[res], params, out)
    return BlockCut(*out)


ClipCut = collections.namedtuple("ClipCut", "held past_caches parts tables")


def clip(P, sizes, dtypes):
    """held: units a thread holds (0: in ranges); parts: ranges whose sums a member's norm is made of; tables: launches a pass."""
    out = (ctypes.c_longlong * 4)()
    _lib().clip((ctypes.c_longlong * len(sizes))(*sizes), (ctypes.c_int * len(sizes))(*[_TYPES[t] for t in dtypes]), len(sizes), P, out)
    return ClipCut(*out)
