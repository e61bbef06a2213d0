"""Host side of the operators around compressed layers: sizes, refusals that need no GPU, constants."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2208_11580_amd import binding

    if not os.path.exists(binding.LIB_PATH):
        from paper_2208_11580_amd import build

        build.build_lib()
    return binding.load_library()


def test_packed_sizes(lib):
    n = ctypes.c_size_t()
    for R, d, group, groups in ((16, 128, 128, 1), (16, 128, 0, 1), (17, 129, 128, 2), (16, 256, 32, 8), (1, 1, 64, 1),
                                (4096, 4096, 128, 32), (4096, 4096, 256, 16), (768, 768, 4096, 1), (100, 100, 100, 1)):
        assert lib.obc_pack4_bytes(R, d, group, ctypes.byref(n)) == 0
        rows, cols = -(-R // 16) * 16, -(-d // 128) * 128
        assert n.value == rows * cols // 2 + 4 * rows * groups, (R, d, group)
    assert lib.obc_pack4_bytes(0, 128, 0, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.obc_pack4_bytes(70000, 131072, 0, ctypes.byref(n)) == 0 and n.value > 2 ** 32
    for R, d, group in ((-1, 8, 0), (8, 0, 0), (8, 200, 48), (8, 200, -32), (8, 500, 129)):
        assert lib.obc_pack4_bytes(R, d, group, ctypes.byref(n)) == -1
    assert lib.obc_pack4_bytes(8, 8, 0, None) == -1


def test_workspace_queries(lib):
    n = ctypes.c_size_t()
    for T in (0, 1, 16, 17, 100, 5000):
        for t in (0, 1, 2, 3):
            assert lib.obc_product4_workspace_bytes(T, 300, 500, 64, t, ctypes.byref(n)) == 0
        for t in (0, 1, 2):
            assert lib.obc_product4_grad_workspace_bytes(T, 300, 500, 64, t, ctypes.byref(n)) == 0
        assert lib.obc_product4_grad_workspace_bytes(T, 300, 500, 64, 3, ctypes.byref(n)) == -1
        assert lib.obc_rmsnorm_grad_workspace_bytes(T, 300, ctypes.byref(n)) == 0
    assert lib.obc_product4_workspace_bytes(-1, 300, 500, 64, 0, ctypes.byref(n)) == -1
    assert lib.obc_product4_workspace_bytes(1, 300, 500, 64, 4, ctypes.byref(n)) == -1
    assert lib.obc_product4_workspace_bytes(1, 300, 500, 40, 0, ctypes.byref(n)) == -1
    assert lib.obc_product4_workspace_bytes(1, 300, 500, 64, 0, None) == -1
    assert lib.obc_rmsnorm_grad_workspace_bytes(1, 0, ctypes.byref(n)) == -1


def test_a_null_context_is_refused(lib):
    p = ctypes.c_void_p(64)
    assert lib.obc_group_grid(None, p, None, 1, 1, 0, 15, 0, p, p) == -1
    assert lib.obc_pack4(None, p, p, p, 1, 1, 0, p) == -1
    assert lib.obc_product4(None, p, 1, 1, 0, p, 0, None, 1, 1, p, 0, 1, None, 0) == -1
    assert lib.obc_product4_grad(None, p, 1, 1, 0, p, 0, 1, 1, p, 1, None, 0) == -1
    assert lib.obc_rmsnorm(None, p, None, 0, p, 0.0, 1, 1, None, p, 0, None, None) == -1
    assert lib.obc_rmsnorm_grad(None, p, p, p, p, None, 0, 1, 1, p, p, None, 0) == -1
    assert lib.obc_distill(None, p, 0, 1, 1, 1, p, p, 1, 1.0, None, p, None, 0) == -1


def test_constants_match_the_header():
    from paper_2208_11580_amd import binding

    text = open(os.path.join(ROOT, "include", "obc.h")).read()
    defs = dict(re.findall(r"#define\s+(OBC_[A-Z0-9_]+)\s+\(?(-?\d+)\)?", text))
    for name in ("F32", "F16", "BF16", "I8", "GRID_SYMMETRIC", "GRID_ZERO"):
        assert int(defs["OBC_" + name]) == getattr(binding, name)
