"""Refusals of the operators that need no handle: nothing here reaches a device."""
import ctypes as C
import os

import pytest

from paper_1711_09846_amd import binding

EINVAL, ENOMEM, EUNSUPPORTED = -1, -2, -5
MEM = 1 << 40      # an address that nothing reads: every call below is refused before it launches anything


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1711_09846_amd import build
        build.build_library(verbose=False)


def _grads(**kw):
    k = dict(d_src=MEM, d_dst=MEM + (1 << 30), len=100, src_stride=128, dst_stride=128, dtype=0, unused=0)
    k.update(kw)
    return (binding.PbtGrad * 1)(binding.PbtGrad(**k))


def _clip(grads, n=1, P=4, max_norm=MEM, stride=1, norm=MEM, work=MEM, work_bytes=1 << 20):
    return binding.lib().pbt_clip_gradients(grads, n, P, max_norm, stride, norm, work, work_bytes, None)


@pytest.mark.parametrize("kw,call,status", [
    (dict(dtype=2), {}, EINVAL), (dict(len=-1), {}, EINVAL), (dict(d_src=0), {}, EINVAL), (dict(d_dst=0), {}, EINVAL),
    (dict(d_src=MEM + 2), {}, EINVAL), (dict(src_stride=99), {}, EINVAL), (dict(dst_stride=99), {}, EINVAL), (dict(unused=1), {}, EINVAL),
    (dict(d_dst=MEM, dst_stride=256), {}, EINVAL),                    # in place with two strides
    (dict(d_dst=MEM + 4 * 50), {}, EINVAL),                           # halves of a member's tensor over one another
    ({}, dict(n=0), EINVAL), ({}, dict(P=0), EINVAL), ({}, dict(P=1025), EINVAL), ({}, dict(stride=-1), EINVAL), ({}, dict(max_norm=MEM + 1), EINVAL),
    ({}, dict(max_norm=None, norm=None), EINVAL), ({}, dict(work=None), EINVAL), ({}, dict(work=MEM + 4), EINVAL), ({}, dict(work_bytes=8), ENOMEM),
])
def test_clip_refusals(kw, call, status):
    assert _clip(_grads(**kw), **call) == status
    assert len(binding.lib().pbt_last_error(None)) > 10


def test_clip_work_bytes():
    n = C.c_size_t()
    assert binding.lib().pbt_clip_work_bytes(_grads(), 1, 4, C.byref(n)) == 0 and 0 < n.value < (1 << 20)
    assert binding.lib().pbt_clip_work_bytes(_grads(len=1 << 40, src_stride=1 << 40), 1, 4, C.byref(n)) == 0 and n.value < (1 << 20)
    assert binding.lib().pbt_clip_work_bytes(_grads(), 1, 4, None) == EINVAL


def _settings(**kw):
    k = dict(rot_dim=64, layout=0, scaling=0, unused=0, base=10000.0, factor=1.0, trained_len=0.0, low=1.0, high=32.0, gain=1.0)
    k.update(kw)
    return binding.PbtRotary(**k)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=514), dict(layout=2), dict(scaling=4), dict(unused=1), dict(base=0.0),
                                dict(base=float("inf")), dict(gain=float("nan")), dict(scaling=1, factor=0.0), dict(scaling=3, factor=2.0),
                                dict(scaling=3, factor=2.0, trained_len=4096.0, low=2.0, high=2.0)])
def test_rotary_settings_refusals(kw):
    assert binding.lib().pbt_rotary_plan(C.byref(_settings(**kw)), MEM, 1 << 20, None) == EINVAL


def test_rotary_plan_table_refusals():
    s = C.byref(_settings())
    assert binding.lib().pbt_rotary_plan(s, None, 1 << 20, None) == EINVAL
    assert binding.lib().pbt_rotary_plan(s, MEM + 4, 1 << 20, None) == EINVAL
    assert binding.lib().pbt_rotary_plan(s, MEM, 255, None) == ENOMEM


def _apply(group=(), table=MEM, n=1, dtype=1, rows=10, width=64, pos=MEM, size=4, start=0, period=0, backward=0):
    g = dict(d_src=MEM, d_dst=MEM + (1 << 30), src_row=1536, src_head=64, dst_row=512, dst_head=64, heads=8, unused=0)
    g.update(group)
    groups = (binding.PbtHeads * 5)(*([binding.PbtHeads(**g)] * 5))
    return binding.lib().pbt_rotary_apply(C.byref(_settings()), table, groups, n, dtype, rows, width, pos, size, start, period, backward, None)


@pytest.mark.parametrize("call", [
    dict(table=None), dict(table=MEM + 1), dict(n=0), dict(n=5), dict(dtype=3), dict(rows=-1), dict(rows=1 << 31), dict(width=62), dict(width=1 << 17), dict(size=2),
    dict(pos=MEM + 2), dict(pos=None, period=-1), dict(pos=None, start=1 << 50), dict(backward=2), dict(group=dict(heads=0)), dict(group=dict(unused=1)),
    dict(group=dict(d_src=0)), dict(group=dict(d_dst=MEM + 1)), dict(group=dict(src_head=63)), dict(group=dict(dst_head=32)), dict(group=dict(dst_row=511)),
    dict(group=dict(src_row=-512)), dict(group=dict(src_row=1 << 40)),
    dict(group=dict(d_dst=MEM)),                                      # the same memory with another row distance
    dict(group=dict(d_dst=MEM + 2 * 64, dst_row=1536)),               # the same rows, one head further
])
def test_rotary_apply_refusals(call):
    assert _apply(**call) == EINVAL


def test_rotary_groups_that_meet_are_refused():
    """The same heads twice, one group's dst over another's src or dst, halves of heads over one another.  (Adjacent heads of one projection in place are
    what test_gpu_operators.py does.)"""
    far = MEM + (1 << 30)
    for a, b in (((MEM, MEM), (MEM, MEM)), ((MEM, far), (far, far)), ((MEM, far), (MEM + 1024, far + 512)), ((MEM, MEM), (MEM + 512, MEM + 512))):
        assert _apply_two(a, b) == EINVAL and b"overlaps group" in binding.lib().pbt_last_error(None), (a, b)


def _apply_two(a, b):
    base = dict(src_row=1536, src_head=64, dst_row=1536, dst_head=64, heads=8, unused=0)
    groups = (binding.PbtHeads * 2)(binding.PbtHeads(**base, d_src=a[0], d_dst=a[1]), binding.PbtHeads(**base, d_src=b[0], d_dst=b[1]))
    return binding.lib().pbt_rotary_apply(C.byref(_settings()), MEM, groups, 2, 1, 10, 64, None, 0, 0, 0, 0, None)


def test_rotary_of_no_rows_is_done():
    assert _apply(rows=0) == 0


def _block(**kw):
    k = dict(rows=10, P=2, d=64, post=1, pre=2, gate=0, gate_act=0, dtype=1, res_dtype=0, eps=1e-5, alpha=1.0, beta=1.0)
    k.update(kw)
    return binding.PbtBlockNorm(**k)


@pytest.mark.parametrize("kw,status", [
    (dict(P=0), EINVAL), (dict(P=1025), EINVAL), (dict(rows=-1), EINVAL), (dict(d=0), EINVAL), (dict(d=8193), EUNSUPPORTED), (dict(post=3), EINVAL), (dict(pre=-1), EINVAL),
    (dict(post=0, pre=0), EINVAL), (dict(gate=3), EINVAL), (dict(gate=1, gate_act=1), EINVAL), (dict(gate_act=5), EINVAL), (dict(dtype=2), EINVAL),
    (dict(res_dtype=-1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(alpha=float("nan")), EINVAL), (dict(beta=float("inf")), EINVAL)])
def test_block_norm_settings_refusals(kw, status):
    n = C.c_size_t()
    assert binding.lib().pbt_block_norm_work_bytes(C.byref(_block(**kw)), C.byref(n)) == status


def _at(k, pitch=64):
    return binding.PbtRows(MEM + (k << 24), pitch)


def _forward(block=(), **kw):
    b = _block(**dict(block))
    a = dict(y=_at(0), x=_at(1), gate=_at(2), params=binding.PbtBlockParams(stride=64), out=_at(3), z=_at(4), stats=MEM)
    a.update(kw)
    ref = lambda v: None if v is None else C.byref(v)  # noqa: E731
    return binding.lib().pbt_block_norm_forward(C.byref(b), ref(a["y"]), ref(a["x"]), ref(a["gate"]), ref(a["params"]), ref(a["out"]), ref(a["z"]), a["stats"], None)


@pytest.mark.parametrize("kw", [
    dict(y=None), dict(x=binding.PbtRows(0, 64)), dict(y=binding.PbtRows(MEM + 1, 64)), dict(x=_at(1, 63)), dict(out=None), dict(z=None), dict(params=None),
    dict(block=dict(gate=1)), dict(block=dict(gate=2), gate=None), dict(stats=MEM + 4), dict(params=binding.PbtBlockParams(post_gain=MEM + 2, stride=64)),
    dict(params=binding.PbtBlockParams(pre_gain=MEM, stride=63)), dict(out=_at(0)), dict(z=_at(1)), dict(z=_at(3)),
    dict(out=binding.PbtRows(MEM + (1 << 24) + 4, 64)),               # one element further than x
    dict(z=_at(0, 72)),                                               # over y with another pitch
])
def test_block_norm_forward_refusals(kw):
    assert _forward(**kw) == EINVAL


def test_block_norm_of_no_rows_is_done():
    assert _forward(block=dict(rows=0), y=None, x=None, out=None, z=None) == 0


def _backward(block=(), **kw):
    b = _block(**dict(block))
    a = dict(y=_at(0), x=_at(1), gate=_at(2), params=binding.PbtBlockParams(gate=MEM, stride=64), stats=MEM, dout=_at(3), dz=_at(4), dy=_at(5), dx=_at(6), dgate=_at(7),
             grads=binding.PbtBlockParams(stride=64), work=MEM, bytes=1 << 24)
    a.update(kw)
    ref = lambda v: None if v is None else C.byref(v)  # noqa: E731
    return binding.lib().pbt_block_norm_backward(C.byref(b), ref(a["y"]), ref(a["x"]), ref(a["gate"]), ref(a["params"]), a["stats"], ref(a["dout"]), ref(a["dz"]),
                                                 ref(a["dy"]), ref(a["dx"]), ref(a["dgate"]), ref(a["grads"]), a["work"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(stats=None), EINVAL), (dict(stats=MEM + 8), EINVAL), (dict(dout=None, dz=None), EINVAL), (dict(block=dict(pre=0), dout=None), EINVAL), (dict(dy=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(block=dict(gate=2), dgate=None), EINVAL), (dict(grads=None), EINVAL), (dict(grads=binding.PbtBlockParams(gate=MEM, stride=64)), EINVAL),
    (dict(block=dict(post=0), grads=binding.PbtBlockParams(post_gain=MEM, stride=64)), EINVAL),
    (dict(block=dict(pre=0), grads=binding.PbtBlockParams(pre_bias=MEM, stride=64)), EINVAL), (dict(work=None), EINVAL), (dict(work=MEM + 8), EINVAL),
    (dict(bytes=16), ENOMEM), (dict(dy=_at(0)), EINVAL), (dict(dx=_at(1)), EINVAL), (dict(dx=_at(5)), EINVAL), (dict(block=dict(gate=2), dgate=_at(4)), EINVAL),
    (dict(dy=_at(4, 80)), EINVAL)])
def test_block_norm_backward_refusals(kw, status):
    assert _backward(**kw) == status


# ---- options of the transformer workload, the clip-norm column ----

def _tf(**options):
    from paper_1711_09846_amd import workloads
    wl = workloads.TRANSFORMER.replace(tf_options=options, **({"n_blocks": 5} if options.get("deep") else {}))
    return wl


def _sizes(wl, **fields):
    o = binding.make_tf_options(wl.replace(tf_options={k: v for k, v in wl.tf_options.items() if k != "deep"}))
    for k, v in fields.items():
        setattr(o, k, v)
    return binding.query_sizes(binding.make_config(wl, 1), o)


def test_transformer_options_layout():
    from paper_1711_09846_amd import workloads
    plain = binding.query_sizes(binding.make_config(workloads.TRANSFORMER, 1))
    assert binding.make_tf_options(workloads.TRANSFORMER) is None
    same = _sizes(_tf(learned_positions=True))
    assert same[:2] == plain[:2] and bytes(same[2]) == bytes(plain[2])
    turned = _sizes(_tf(rotary=dict(rot_dim=64), learned_positions=False))
    assert bytes(turned[2]) == bytes(plain[2]) and turned[0] - plain[0] == 2048
    wl = _tf(block_norm="rms", alpha=0.9, beta=0.5)
    lay = _sizes(wl)[2]
    shapes = workloads.transformer_shapes(wl)
    assert lay.n_seg == len(shapes) == 2 + 16 * wl.n_blocks + 4
    assert [lay.seg_len[j] for j in range(lay.n_seg)] == [a[0] * (a[1] if len(a) > 1 else 1) for a in shapes]
    assert lay.n_params == plain[2].n_params + 4 * wl.n_blocks * wl.d_model
    assert _sizes(_tf(block_norm="layer", deep=True))[2].n_seg == 2 + 16 * 5 + 4


@pytest.mark.parametrize("options,fields,status", [
    (dict(rotary=dict(rot_dim=66)), {}, EINVAL), (dict(rotary=dict(rot_dim=64)), dict(rotary=2), EINVAL), (dict(learned_positions=True), dict(learned_positions=2), EINVAL),
    (dict(block_norm="rms"), dict(block_norm=3), EINVAL), (dict(block_norm="rms"), dict(unused=1), EINVAL), (dict(block_norm="rms"), dict(beta=float("nan")), EINVAL),
    (dict(learned_positions=True), dict(alpha=0.5), EINVAL), (dict(rotary=dict(rot_dim=64, base=-1.0)), {}, EINVAL)])
def test_transformer_options_refusals(options, fields, status):
    with pytest.raises(binding.PbtError) as e:
        _sizes(_tf(**options), **fields)
    assert e.value.status == status


def test_transformer_options_need_their_workload_and_sizes():
    from paper_1711_09846_amd import workloads
    o = binding.make_tf_options(_tf(block_norm="rms"))
    for wl, status in ((workloads.MLP_WIDE, EINVAL), (_tf(block_norm="rms").replace(n_blocks=6), EUNSUPPORTED),
                       (_tf(block_norm="rms").replace(d_model=2056, heads=1, n_blocks=1), EUNSUPPORTED)):
        with pytest.raises(binding.PbtError) as e:
            binding.query_sizes(binding.make_config(wl, 1), o)
        assert e.value.status == status


def test_clip_norm_column():
    from paper_1711_09846_amd import workloads as W
    def with_clip(wl, **kw):
        return binding.make_config(wl.replace(roles=wl.roles + [W.ROLE_CLIP_NORM], h_max=wl.h_max + [float("inf")], priors=wl.priors + [("log", 0.1, 1.0)]), 1, **kw)
    for wl in (W.MLP_WIDE, W.TRANSFORMER, W.A2C_MLP):
        plain, clip = binding.query_sizes(binding.make_config(wl, 1)), binding.query_sizes(with_clip(wl))
        assert bytes(plain[2]) == bytes(clip[2]) and clip[0] > plain[0] and clip[1] > plain[1]
    for wl, kw in ((W.MLP_SMALL, {}), (W.GAN_MLP, {}), (W.MLP_WIDE, dict(fuse_optimizer=1))):
        with pytest.raises(binding.PbtError) as e:
            binding.query_sizes(with_clip(wl, **kw))
        assert e.value.status == EUNSUPPORTED
