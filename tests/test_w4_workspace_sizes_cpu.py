"""mlpmoe_w4_workspace_bytes is 0 for exactly the sizes that the forward on 4-bit weights refuses."""
import ctypes

import numpy as np
import pytest

from paper_2511_21089_amd import binding as mm

P = ctypes.c_void_p(0x1000)
MOST = 65535 * 16


def accepted(T, d_model, d_inter, B):
    """Whether the forward gets as far as its workspace (none is given, so nothing is enqueued) or has nothing to do."""
    off = np.full(B + 1, d_inter, np.int32)
    off[0] = 0
    al, mk = np.ones(B, np.float32), np.ones(B, np.uint8)
    rc = mm.lib.mlpmoe_forward_w4_ws(P, P, P, P, P, P, P, off.ctypes.data, al.ctypes.data, mk.ctypes.data, None, T, d_model, d_inter, B, 2,
                                     P, None, 0, None)
    assert rc in (mm.ERR_WORKSPACE, mm.OK, mm.ERR_SHAPE, mm.ERR_UNSUPPORTED), rc
    return rc in (mm.ERR_WORKSPACE, mm.OK)


@pytest.mark.parametrize("T", [-1, 0, 1, 16, 17, 4096, MOST, MOST + 1, 1 << 24, 2 ** 31 - 1])
def test_zero_for_what_is_refused(T):
    for d_model in (-32, 0, 1, 31, 32, 48, 64, 100, 4096, 131072, 131072 + 32, 1 << 22, 2 ** 31 - 1):
        for d_inter in (-32, 31, 32, 96, 100, 14336, 131072, 131072 + 32, 1 << 22, 2 ** 31 - 32, 2 ** 31 - 1):
            n = mm.mlpmoe_w4_workspace_bytes(T, d_model, d_inter, 2)
            assert (n > 0) == accepted(T, d_model, d_inter, 2), (T, d_model, d_inter, n)
            assert n < 1 << 40


def test_limits_of_branches_and_layers_without_neurons():
    f = mm.mlpmoe_w4_workspace_bytes
    assert f(4, 64, 0, 1) > 0 and f(4, 64, 64, 64) > 0
    assert f(4, 64, 64, 0) == 0 and f(4, 64, 64, 65) == 0 and f(4, 64, 64, -1) == 0
