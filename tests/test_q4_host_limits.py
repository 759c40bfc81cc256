"""The 4-bit cache's entry points without a GPU: the limits of what attention takes, calls that ask for nothing."""
import ctypes as C

import pytest
import torch

from paper_2508_15806_b200 import binding as B
from test_q4_host import FAKE, L, attend_params, cache          # noqa: F401


def test_a_scale_that_leaves_the_products_range_is_refused(L):  # noqa: F811
    # scores are formed in units of 2^-73 / scale: 2^73 * 2^54 * log2(e) is the last power of two below fp32's end
    f, c = C.c_void_p(FAKE), C.byref(cache())
    for scale in (2.0 ** 54 * 1.001, -2.0 ** 55, 3e38, float("inf")):
        p = C.byref(attend_params(scale=scale))
        assert L.slkv_q4_attend_workspace_bytes(c, p, 0) == 0, scale
        assert L.slkv_q4_attend(c, p, f, None, None, f, None, 0, None, f, 1 << 40, None) == B.ERR["BAD_SHAPE"], scale
    for scale in (2.0 ** 54, -2.0 ** 54, 0.0, 1e-38):
        assert L.slkv_q4_attend_workspace_bytes(c, C.byref(attend_params(scale=scale)), 0) > 0, scale
