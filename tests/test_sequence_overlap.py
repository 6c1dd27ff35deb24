"""Outputs of the window, convolution and scan calls over every other tensor of the call, refused before any launch (no GPU needed)."""
import ctypes

import pytest

import paper_2606_09862_amd as bla
from test_window_abi import INVALID, MUCH, WS, addresses, lib  # noqa: F401

FAR = 0x9000000000
WINDOW = (2, 4, 2, 100, 64, 50, 4, 1, 0, 0.0)
CONV = (2, 4, 100, 64, 4, 1, 1)
SSM = (2, 4, 2, 100, 64, 64, 1)
# name: parameters, tensors before the workspace, outputs, whether a workspace follows, input that an output may be (in place)
CALLS = {
    "bla_window_forward": (bla.WindowParams(*WINDOW), 11, (7, 8, 9, 10), True, None),
    "bla_window_step": (bla.WindowParams(*WINDOW), 7, (4, 5, 6), True, None),
    "bla_window_backward": (bla.WindowParams(*WINDOW), 10, (7, 8, 9), True, None),
    "bla_conv_forward": (bla.ConvParams(*CONV), 7, (5, 6), False, None),
    "bla_conv_step": (bla.ConvParams(*CONV), 6, (4, 5), False, (3, 5)),
    "bla_conv_backward": (bla.ConvParams(*CONV), 11, (7, 8, 9, 10), True, None),
    "bla_ssm_forward": (bla.SsmParams(*SSM), 10, (8, 9), True, None),
    "bla_ssm_step": (bla.SsmParams(*SSM), 9, (7, 8), False, (6, 8)),
    "bla_ssm_backward": (bla.SsmParams(*SSM), 17, (10, 11, 12, 13, 14, 15, 16), True, None),
}


@pytest.mark.parametrize("name", CALLS)
def test_outputs_over_other_tensors(lib, name):  # noqa: F811
    p, n, outputs, room, in_place = CALLS[name]
    for o in outputs:
        for i in range(n):
            if i == o or in_place in ((i, o), (o, i)):
                continue
            a = addresses(n)
            a[i] = a[o] = ctypes.c_void_p(FAR)
            tail = (WS, MUCH) if room else ()
            assert getattr(lib, name)(ctypes.byref(p), *a, *tail, None) == INVALID, (o, i)
