"""Settings that would be taken for others: nothing here reaches a device."""
import ctypes as C
import os

import pytest

from paper_1711_09846_amd import binding, workloads as W

EINVAL = -1


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1711_09846_amd import build
        build.build_library(verbose=False)


@pytest.mark.parametrize("options", [dict(learned_position=False), dict(rotary=dict(rot_dim=64), blocknorm="rms")])
def test_unknown_transformer_options_are_refused(options):
    with pytest.raises(ValueError, match="tf_options"):
        binding.make_tf_options(W.TRANSFORMER.replace(tf_options=options))


def _settings(**kw):
    k = dict(rot_dim=4, layout=0, scaling=0, unused=0, base=10000.0, factor=1.0, trained_len=0.0, low=1.0, high=32.0, gain=1.0)
    k.update(kw)
    return binding.PbtRotary(**k)


@pytest.mark.parametrize("kw", [
    dict(scaling=1, factor=1e-310), dict(base=1e-300, rot_dim=64, scaling=1, factor=1e-20),      # frequencies past the doubles
    dict(scaling=2, factor=1e200),                                                               # a base past them: 10000 (1e200)^2
    dict(scaling=3, factor=1e-310, trained_len=1e-300), dict(gain=1e39)])                        # a gain past the floats
def test_rotary_settings_out_of_range_are_refused(kw):
    assert binding.lib().pbt_rotary_plan(C.byref(_settings(**kw)), 1 << 40, 1 << 20, None) == EINVAL
    if "rot_dim" not in kw:
        wl = W.TRANSFORMER.replace(tf_options=dict(rotary=dict(rot_dim=4)))
        o = binding.make_tf_options(wl)
        o.rot = _settings(**kw)
        with pytest.raises(binding.PbtError) as e:
            binding.query_sizes(binding.make_config(wl, 1), o)
        assert e.value.status == EINVAL
