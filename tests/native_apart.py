"""The entry points' check of memory that meets (csrc/operators_apart.h), compiled for the host."""
import ctypes
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1711_09846_amd", "csrc")
_SOURCE = r"""
#include "operators_apart.h"
// fields: [n][5] address, bytes, stride, count, written; returns 0 (apart) or 1 + the pair in out
extern "C" int meeting(const long long* fields, int n, int* out) {
  pbt::Region* r = new pbt::Region[n];
  for (int k = 0; k < n; ++k) r[k] = pbt::Region{(uintptr_t)fields[5 * k], fields[5 * k + 1], fields[5 * k + 2], fields[5 * k + 3], fields[5 * k + 4] != 0, k};
  pbt::RegionKey* keys = new pbt::RegionKey[n];
  const bool found = pbt::find_meeting(r, keys, n, out, out + 1);
  delete[] r;
  delete[] keys;
  return found;
}
// fields: address, row, head, rows, heads, width of both
extern "C" int heads_apart(const long long* f) {
  const auto view = [](const long long* v) { return pbt::HeadView{(uintptr_t)v[0], v[1], v[2], v[3], v[4], v[5]}; };
  return pbt::heads_apart(view(f), view(f + 6));
}
"""


@functools.lru_cache(None)
def _lib():
    d = tempfile.mkdtemp()
    src, so = os.path.join(d, "apart.cpp"), os.path.join(d, "apart.so")
    with open(src, "w") as f:
        f.write(_SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
    return ctypes.CDLL(so)


def meeting(regions):
    """regions: (address, bytes, stride, count, written); the indices of two that meet, one of them written, or None."""
    flat = [int(v) for r in regions for v in r]
    out = (ctypes.c_int * 2)()
    return tuple(out) if _lib().meeting((ctypes.c_longlong * len(flat))(*flat), len(regions), out) else None


def heads_apart(a, b):
    """a, b: (address, row, head, rows, heads, width) in bytes."""
    return bool(_lib().heads_apart((ctypes.c_longlong * 12)(*a, *b)))
