"""Where the calls of the 4-bit cache end: sizes that a launch cannot have are refused (CPU: the pointers are fake)."""
import ctypes as ct

import pytest

from tests.test_mx_refusals import Calls


@pytest.fixture(scope="module")
def mk():
    from paper_2510_09309_amd import binding
    return binding


def test_more_workgroups_than_a_launch_can_have(mk):
    """A launch has fewer than 2^32 threads along a dimension: 65535 heads of 257 workgroups of 256 threads are more."""
    c = Calls(mk, H=65535, d=64, dtype=mk.MASKKV_F32, n_resp=257 * 32, P_max=100)
    size = ct.c_size_t()
    assert c.lib.maskkv_attend_mx_workspace_bytes(ct.byref(c.desc), ct.c_int64(10), ct.byref(size)) == 0
    assert c.attend(ws=1 << 20, ws_bytes=1 << 62) == 2 and "workgroups" in c.error()
