"""The scales that ssd.h names, and no others, are taken."""
import ctypes
import os
import re

import pytest

from paper_2603_09555_amd import build, ssd
from test_block_abi import FAKE, shape


@pytest.mark.parametrize("name", ["ssd_attn_step", "ssd_attn_prefill"])
def test_the_range_is_the_header_s(name):
    text = open(os.path.join(build.INCLUDE, "ssd.h")).read()
    most = [float(m) for m in re.findall(r"\* +scale +positive, up to (\S+)", text)]
    assert most == [1e30, 1e30]
    s, cu = shape(), [FAKE] if name == "ssd_attn_prefill" else []
    need = ctypes.c_size_t(getattr(ssd, name[4:] + "_workspace_bytes")(s))

    def call(scale):   # (without a y, which is looked at behind the scale)
        return getattr(ssd.raw(), name)(ctypes.byref(s), *cu, FAKE, FAKE, FAKE, FAKE, FAKE, ctypes.c_float(scale), None, FAKE, need, None)

    for scale in (1e-45, 1e-30, 0.1, 1.0, 9.9e29):
        assert call(scale) == -1, scale
    for scale in (1.1e30, 3e38, float("inf"), float("nan"), 0.0, -1e-45, -1.0):
        assert call(scale) == -2, scale
