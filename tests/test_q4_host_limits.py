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


def test_an_empty_list_of_slots_asks_for_nothing(monkeypatch):
    # the library and the device taken away: a call that gets through is seen
    calls = []
    monkeypatch.setattr(B, "_current_device", lambda: -1)
    monkeypatch.setattr(B, "_fn", {"slkv_q4_unpack": lambda *a: calls.append(a) or B.SLKV_OK})
    t = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt)        # noqa: E731
    c = B.make_q4_cache(t(10, 160, dt=torch.uint8), t(10), None, t(9), t(8), 4)
    c.index = -1
    rows = torch.zeros(10, 128)
    B.slkv_q4_unpack(c, rows[:0], rows[:0], slots=t(0))
    assert calls == []
    with pytest.raises(AssertionError):                             # still looked at
        B.slkv_q4_unpack(c, rows[:0], rows[:0], slots=t(1))
    with pytest.raises(AssertionError):
        B.slkv_q4_unpack(c, rows[:0], rows[:0])
    B.slkv_q4_unpack(c, rows[:1], rows[:1], slots=t(1))
    B.slkv_q4_unpack(c, rows, rows)
    assert len(calls) == 2
