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
