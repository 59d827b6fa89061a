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


def test_heads_count_weights_as_the_blob(lib):
    import synth
    from paper_2608_16329_amd import binding as b
    for hidden, lmax, k in ((1, 0, 16), (4, 3, 32), (8, 5, 64)):
        hp = synth.HParams(n_species=3, lmax=lmax, k=k, reg_hidden=hidden)
        p = b.mlip_heads_params(3, (lmax + 1) * k, hidden, 1, b.MLIP_F32, (lmax + 1) * k)
        one = synth.HParams(n_species=3, lmax=lmax, k=k, reg_hidden=hidden, reg_cond=0)
        per_head = (synth.weight_count(hp) - synth.weight_count(one)) // 2
        assert b.mlip_heads_weight_count(p) == 3 * per_head
    for bad in ((0, 128, 4), (257, 128, 4), (3, 0, 4), (3, 1025, 4), (3, 128, 0), (3, 128, 9)):
        assert b.mlip_heads_weight_count(b.mlip_heads_params(*bad, 1, 0, 2000)) == 0


def test_adamw_entries_refuse(lib):
    from paper_2608_16329_amd import binding as b
    lib.mlip_adamw_destroy(None)
    assert lib.mlip_heads(None, None, 1, *[None] * 10) == -1
    assert lib.mlip_adamw_step(None, None, None, None, 0) == -1
    assert lib.mlip_adamw_moments(None, None, None, None) == -1
    plan = ctypes.c_void_p()
    one = b.mlip_adamw_tensor(16, None, 16, 4, b.MLIP_F32, b.MLIP_F32, 1)
    for tensors, n, bits, why in ((None, 1, 32, b"no tensors"), (one, 0, 32, b"no tensors"), (one, 1, 16, b"state_bits"),
                                  (b.mlip_adamw_tensor(16, None, None, 4, 0, 0, 1), 1, 32, b"NULL"),
                                  (b.mlip_adamw_tensor(16, None, 16, -1, 0, 0, 1), 1, 32, b"elements"),
                                  (b.mlip_adamw_tensor(16, None, 16, 4, 5, 0, 1), 1, 8, b"dtype")):
        arg = ctypes.byref(tensors) if tensors is not None else None
        assert lib.mlip_adamw_create(arg, n, bits, None, ctypes.byref(plan)) == -1
        assert why in lib.mlip_adamw_last_error(None)
        assert plan.value is None
    two = (b.mlip_adamw_tensor * 2)(one, b.mlip_adamw_tensor(16, 16, 16, 4, 0, 0, 1))
    assert lib.mlip_adamw_create(two, 2, 32, None, ctypes.byref(plan)) == -1
    assert b"into_dev" in lib.mlip_adamw_last_error(None)
