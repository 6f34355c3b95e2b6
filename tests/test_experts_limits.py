"""Sizes that the layers refuse before they touch the GPU (no GPU).

Kernels count rows in 32 bits, round them up to tiles and look ahead by up to some hundred: from 1,023 below
the largest such number on, a row's number would wrap around and pass its test against the end."""
import ctypes

import pytest

from paper_1801_01554_gb300 import bp, build

MOST = 2 ** 31 - 1 - 1023
P = 0x10000   # an address that is never read


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(bp.lib_path()):
        build.build()
    return bp.load()


@pytest.mark.parametrize("create,args", [
    ("bp_router_create", (8, 1, 0, MOST + 1, 0)), ("bp_router_create", (8, 1, 0, 2 ** 31 - 1, 0)),
    ("bp_router_create", (8, 3, 0, MOST // 3 + 1, 0)), ("bp_experts_create", (2, 8, 8, 0, MOST + 1)),
    ("bp_experts_create", (2, 8, 8, 1, 2 ** 31 - 1)), ("bp_adapters_create", (2, 4, 8, 8, 0, MOST // 128 + 1, 1)),
    ("bp_adapters_create", (2, 4, 8, 8, 1, 1, MOST + 1))])
def test_handles_for_more_rows_than_can_be_counted(lib, create, args):
    out = ctypes.c_void_p()
    assert getattr(lib, create)(*args, ctypes.byref(out)) == bp.BP_EINVAL
    assert out.value is None and b"must be in [1, " in lib.bp_last_error()


@pytest.mark.parametrize("n,k", [(MOST + 1, 1), (2 ** 31 - 1, 1), (MOST // 16 + 1, 16)])
def test_mixes_of_more_patterns_than_can_be_counted(lib, n, k):
    assert lib.bp_mix(P, 4, P, P, n, k, 8, 0, P, None) == bp.BP_EINVAL
    assert lib.bp_mix_backward(P, P, 4, P, P, n, k, 8, 0, P, P, None) == bp.BP_EINVAL
