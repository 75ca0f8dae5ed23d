"""The workspace of readme_verify_drafts, on the CPU: a request's state is in its
workgroup, so none is asked for, and a call needs none."""
import ctypes

import pytest

from tests.test_abi_drafts import FAKE, _verify, lib  # noqa: F401


@pytest.mark.parametrize("T,R,V", [(1, 1, 1), (16, 2, 1000), (16, 2, 100000), (1 << 27, 1 << 20, 1 << 16),
                                   (1 << 20, 32, (1 << 31) - 1), (0, 0, 1)])
def test_none_is_needed(lib, T, R, V):  # noqa: F811
    assert lib.readme_verify_drafts_workspace_bytes(T, R, V) == 0


def test_a_call_passes_without_one(lib):  # noqa: F811
    """No workspace is no error: what is refused here is another argument, checked
    after it, and a call of nothing."""
    for ws, size in ((None, 0), (FAKE, 0), (FAKE, 1 << 40)):
        assert _verify(lib, ws=ws, wsb=size, T=0, R=0) == 0
        assert _verify(lib, ws=ws, wsb=size, token=None) == 1
    assert _verify(lib, ws=ctypes.c_void_p(4100), wsb=64) == 1
