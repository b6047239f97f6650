"""CPU checks of the microscaled 4-bit and mixture entry points at the edges of
what they accept: each line is refused, or answered rightly, by both the C calls
and their binding."""
import pytest

from test_abi import ss  # noqa: F401  (fixture: the built library)
from test_mx4_abi import BIG, FAKE, groups, status


def refused(ss, want, f, *args, **named):  # noqa: F811
    with pytest.raises(ss.SwiftSpecError) as e:
        f(*args, **named)
    assert e.value.status == want


def test_router_workspace_alignment(ss):  # noqa: F811
    """The counts of the router's second launch are read eight bytes at a time."""
    lib = ss.lib()
    for off in (1, 2, 4, 6, 12):
        assert status(lib, "moe_route", FAKE, 8, 1, FAKE, FAKE, groups(ss), FAKE + off, BIG) == ss.MISALIGNED
        assert status(lib, "moe_group", FAKE, groups(ss), FAKE + off, BIG) == ss.MISALIGNED
    small = lib.swiftspec_moe_route_workspace_bytes(4, 8, 2) - 1
    for off in (0, 8):  # aligned enough: the next check answers
        assert status(lib, "moe_route", FAKE, 8, 1, FAKE, FAKE, groups(ss), FAKE + off, small) == ss.WORKSPACE_TOO_SMALL
        assert status(lib, "moe_group", FAKE, groups(ss), FAKE + off, small) == ss.WORKSPACE_TOO_SMALL
