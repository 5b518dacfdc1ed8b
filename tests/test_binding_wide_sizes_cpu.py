"""The workspace sizes of the router and of the 4-bit weights for numbers that do not fit the library's 32-bit arguments: none, not
those of the lower 32 bits."""
import pytest

from paper_2511_21089_amd import binding as mm


@pytest.mark.parametrize("far", [1 << 31, (1 << 32) + 16, 1 << 40, -(1 << 32) + 16, -(1 << 31) - 1])
def test_sizes_past_32_bits(far):
    assert mm.mlpmoe_route_workspace_bytes(16, 16) > 0 and mm.mlpmoe_w4_workspace_bytes(16, 64, 64, 16) > 0
    for i in range(2):
        a = [16, 16]
        a[i] = far
        assert mm.mlpmoe_route_workspace_bytes(*a) == 0, a
    for i in range(4):
        a = [16, 64, 64, 16]
        a[i] = far if i in (0, 3) else far + 48
        assert mm.mlpmoe_w4_workspace_bytes(*a) == 0, a
