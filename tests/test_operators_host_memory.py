"""Refusals of calls whose arguments share memory: nothing here reaches a device."""
import ctypes as C
import os

import pytest

from paper_1711_09846_amd import binding

EINVAL = -1
MEM = 1 << 40      # an address that nothing reads: every call below is refused before it launches anything
FAR = 1 << 30


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1711_09846_amd import build
        build.build_library(verbose=False)


def _error():
    return binding.lib().pbt_last_error(None).decode()


def _clip(*tensors, P=4, max_norm=MEM + 5 * FAR, stride=1, norm=MEM + 6 * FAR, work=MEM + 7 * FAR, work_bytes=1 << 20):
    grads = (binding.PbtGrad * len(tensors))(*[binding.PbtGrad(src, dst, n, pitch, pitch, dtype, 0) for src, dst, n, pitch, dtype in tensors])
    return binding.lib().pbt_clip_gradients(grads, len(tensors), P, max_norm, stride, norm, work, work_bytes, None)


@pytest.mark.parametrize("tensors", [
    [(MEM, MEM + FAR, 100, 128, 0), (MEM + 2 * FAR, MEM, 100, 128, 0)],                     # a dst over another tensor's src
    [(MEM, MEM + FAR, 100, 128, 0), (MEM + 2 * FAR, MEM + FAR, 100, 128, 0)],               # two tensors into one
    [(MEM, MEM, 100, 128, 0), (MEM, MEM + FAR, 100, 128, 0)],                               # clipped in place and read by another
    [(MEM, MEM, 100, 128, 0), (MEM + 4 * 99, MEM + 4 * 99, 29, 128, 0)],                    # columns that share an element
    [(MEM, MEM, 100, 128, 0), (MEM + 4 * 100, MEM + 4 * 100, 29, 128, 0)],                  # the second's rows end in the first's next ones
    [(MEM, MEM, 100, 128, 0), (MEM + 4 * 128 * 3, MEM + 4 * 128 * 3, 10, 16, 1)],           # the first's last row, another type and distance
    [(MEM + 512 * k, MEM + 512 * k, 128, 128 * 100, 0) for k in range(100)] + [(MEM + 2 * FAR, MEM + 512 * 50 + 4, 1, 128 * 100, 0)]])
def test_clip_tensors_that_meet_are_refused(tensors):
    assert _clip(*tensors) == EINVAL and "overlap" in _error()


@pytest.mark.parametrize("kw", [
    dict(norm=MEM + 5 * FAR), dict(norm=MEM + 5 * FAR + 12), dict(max_norm=MEM + 6 * FAR - 8, stride=1),      # norms over bounds that others still read
    dict(norm=MEM + FAR + 4 * 127 + 4 * 128 - 8), dict(norm=MEM + 4), dict(max_norm=MEM + FAR + 400 - 4),                  # in a tensor
    dict(max_norm=MEM + FAR + 400 - 4, stride=128), dict(work=MEM + FAR), dict(work=MEM), dict(work=MEM + 6 * FAR), dict(work=MEM + 5 * FAR),
    dict(max_norm=None, norm=MEM + 8), dict(max_norm=None, work=MEM + 8)])
def test_clip_norms_bounds_and_working_memory_that_meet_are_refused(kw):
    assert _clip((MEM, MEM + FAR, 100, 128, 0), **kw) == EINVAL and "overlap" in _error()


def _at(k, pitch=64):
    return binding.PbtRows(MEM + (k << 24), pitch)


def _place(k):
    return MEM + ((16 + k) << 24)


def _settings(**kw):
    k = dict(rows=10, P=2, d=64, post=1, pre=2, gate=0, gate_act=0, dtype=1, res_dtype=0, eps=1e-5, alpha=1.0, beta=1.0)
    k.update(kw)
    return binding.PbtBlockNorm(**k)


def _forward(n, stats=_place(0), params=None, **kw):
    a = dict(y=_at(0), x=_at(1), gate=_at(2), out=_at(3), z=_at(4))
    a.update(kw)
    return binding.lib().pbt_block_norm_forward(C.byref(n), *[C.byref(a[k]) for k in ("y", "x", "gate")], C.byref(params or binding.PbtBlockParams(stride=64)), C.byref(a["out"]),
                                                C.byref(a["z"]), stats, None)


def _backward(n, stats=_place(0), params=None, grads=None, work=_place(1), **kw):
    a = dict(y=_at(0), x=_at(1), gate=_at(2), dout=_at(3), dz=_at(4), dy=_at(5), dx=_at(6), dgate=_at(7))
    a.update(kw)
    none = binding.PbtBlockParams(stride=64)
    return binding.lib().pbt_block_norm_backward(C.byref(n), *[C.byref(a[k]) for k in ("y", "x", "gate")], C.byref(params or none), stats,
                                                 *[C.byref(a[k]) for k in ("dout", "dz", "dy", "dx", "dgate")], C.byref(grads or none), work, 1 << 24, None)


def _params(stride=64, **kw):
    return binding.PbtBlockParams(stride=stride, **kw)


@pytest.mark.parametrize("kw", [
    dict(stats=_at(0).d), dict(stats=_at(3).d + 16), dict(stats=_at(4).d), dict(params=_params(post_gain=_place(0) + 64)),     # statistics over matrices and a parameter
    dict(params=_params(pre_bias=_at(3).d + 64)), dict(params=_params(pre_gain=_at(4).d)),                                       # outputs over parameters
    dict(n=_settings(gate=1), params=_params(gate=_at(4).d + 64, stride=128))])
def test_block_norm_forward_statistics_and_parameters_that_meet_outputs_are_refused(kw):
    kw = dict(kw)
    assert _forward(kw.pop("n", _settings()), **kw) == EINVAL and "overlap" in _error()


@pytest.mark.parametrize("kw", [
    dict(grads=_params(post_gain=_place(2), pre_gain=_place(2))), dict(grads=_params(post_gain=_place(2), pre_bias=_place(2) + 252)),
    dict(grads=_params(post_gain=_place(2), post_bias=_place(2) + 4 * 96, stride=128)),                      # rows that run into the next member's
    dict(params=_params(pre_gain=_place(2)), grads=_params(pre_gain=_place(2))),                             # over the parameter
    dict(grads=_params(pre_gain=_at(4).d)), dict(grads=_params(pre_gain=_at(6).d)), dict(grads=_params(pre_gain=_place(0))), dict(grads=_params(pre_gain=_place(1))),
    dict(work=_at(0).d), dict(work=_at(6).d), dict(work=_place(0)), dict(stats=_at(5).d), dict(params=_params(pre_gain=_at(5).d)),
    dict(n=_settings(rows=0), grads=_params(post_gain=_place(2), pre_gain=_place(2)))])
def test_block_norm_backward_gradients_and_working_memory_that_meet_are_refused(kw):
    kw = dict(kw)
    assert _backward(kw.pop("n", _settings()), **kw) == EINVAL and "overlap" in _error()


def _rotary(rows, dtype=0, **kw):
    g = dict(d_src=MEM, d_dst=MEM, src_row=64, src_head=64, dst_row=64, dst_head=64, heads=1, unused=0)
    g.update(kw)
    s = binding.PbtRotary(64, 0, 0, 0, 10000.0, 1.0, 0.0, 1.0, 32.0, 1.0)
    return binding.lib().pbt_rotary_apply(C.byref(s), MEM + FAR, (binding.PbtHeads * 1)(binding.PbtHeads(**g)), 1, dtype, rows, 64, None, 0, 0, 0, 0, None)


@pytest.mark.parametrize("kw", [dict(src_row=1 << 31, dst_row=64, d_dst=MEM + (1 << 50)), dict(src_row=1 << 31, dst_row=1 << 31), dict(src_row=64, dst_row=1 << 31, d_dst=MEM + 4)])
def test_rotary_rows_that_span_more_than_addresses_are_refused(kw):
    """2^31 rows, 2^31 elements of 4 bytes apart: 2^64 bytes."""
    assert _rotary((1 << 31) - 1, **kw) == EINVAL and "2^46" in _error()


def _rotary_reads(positions, table=MEM + FAR, dst_row=64, rows=100):
    heads = (binding.PbtHeads * 1)(binding.PbtHeads(MEM, MEM, dst_row, 64, dst_row, 64, 1, 0))
    s = binding.PbtRotary(64, 0, 0, 0, 10000.0, 1.0, 0.0, 1.0, 32.0, 1.0)
    return binding.lib().pbt_rotary_apply(C.byref(s), table, heads, 1, 0, rows, 64, positions, 4, 0, 0, 0, None)


@pytest.mark.parametrize("kw", [dict(positions=MEM), dict(positions=MEM + 100 * 256 - 4), dict(positions=MEM - 4), dict(positions=MEM + 256, dst_row=128), dict(positions=None, table=MEM + 512)])
def test_rotary_positions_and_table_under_the_heads_are_refused(kw):
    assert _rotary_reads(**kw) == EINVAL and "overlap" in _error()
