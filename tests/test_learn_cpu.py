"""Host-side checks of the learning operators' C entries that need no GPU: bad
arguments are answered with a status before anything touches a device."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(os.path.join(ROOT, "paper_2608_16329_amd", "libmlip.so")):
        from paper_2608_16329_amd import build
        build.build()
    from paper_2608_16329_amd import binding
    return binding._lib


def test_null_context_is_safe(lib):
    assert isinstance(lib.mlip_learn_last_error(None), bytes)
    lib.mlip_learn_destroy(None)
    assert lib.mlip_learn_create(None, None) == -1
    assert b"NULL" in lib.mlip_learn_last_error(None)
    size = ctypes.c_size_t()
    assert lib.mlip_learn_memory_bytes(None, ctypes.byref(size)) == -1
    assert lib.mlip_route(None, None, 1, *[None] * 7) == -1
    assert lib.mlip_route_backward(None, None, 1, *[None] * 8) == -1
    assert lib.mlip_group(None, 1, 1, None, None, None) == -1
