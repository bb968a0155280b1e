"""The shapes of tests/test_gpu_w4_forms.py reach every form of the 4-bit product that its plan can choose on 256 CUs, so
that none goes untested when a threshold moves. CPU only."""
import ctypes
import itertools
import os
import random

import pytest

from test_gpu_w4_forms import FORMS

fb = pytest.importorskip("paper_2608_15602_amd.fluxbin")
CUS = 256


class Plan(ctypes.Structure):   # fluxbin::W4Plan
    _fields_ = [("many", ctypes.c_bool), ("nw", ctypes.c_int), ("bt", ctypes.c_int), ("rt", ctypes.c_int),
                ("parts", ctypes.c_int), ("ws_bytes", ctypes.c_uint64)]


@pytest.fixture(scope="module")
def form():
    if not os.path.exists(fb.LIB_PATH):
        pytest.fail("libfluxbin.so is not built; run `python -m paper_2608_15602_amd.build`")
    plan = getattr(fb.lib(), "_ZN7fluxbin7w4_planERK16fluxbin_w4_shapeii")   # fluxbin::w4_plan(shape, B, cus)
    plan.restype, plan.argtypes = Plan, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]

    def of(M, N, g, B):
        """What tells one kernel instance, and whether its sums go through memory, apart."""
        s = fb.W4Shape(M, N, g, 1, 0)
        p = plan(ctypes.addressof(s), B, CUS)
        scales = 128 // g if g < 128 and g < N else 1
        if p.many:
            return "many", p.bt, p.parts > 1, scales
        return p.nw, 1 if B <= 4 else 4 * p.bt, p.rt, p.parts > 1, scales

    return of


def test_every_form_is_tested(form):
    tested = {form(M, N, g, B) for M, N, batches in FORMS for B in batches for g in (32, 64, 128)}
    M = [1, 16, 33, 100, 256, 520, 1024, 2048, 4096, 5904, 8160, 8179, 8192, 8200, 11008, 16384, 16400, 28672]
    N = [64, 130, 260, 520, 1100, 2100, 2600, 4096, 5000, 8192, 14400, 28700]
    B = [1, 2, 4, 5, 16, 17, 32, 33, 48, 49, 64, 65, 100, 128, 256, 512, 1024, 4096, 8192]
    seen = {}
    for m, n, b, g in itertools.product(M, N, B, (32, 64, 128)):
        seen.setdefault(form(m, n, g, b), (m, n, b, g))
    rng = random.Random(1)
    for _ in range(20000):
        m, n, b = (int(2 ** rng.uniform(0, top)) for top in (17, 16, 13))
        g = rng.choice([32, 64, 128])
        seen.setdefault(form(m, n, g, b), (m, n, b, g))
    assert not {k: v for k, v in seen.items() if k not in tested}


def _workspace():
    f = getattr(fb.lib(), "_ZN7fluxbin12w4_workspaceERK16fluxbin_w4_shapeii")   # fluxbin::w4_workspace(shape, B, cus)
    f.restype, f.argtypes = ctypes.c_uint64, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    return f


def test_workspace_serves_every_smaller_batch(form):
    """The workspace of B rows holds what the plan of any batch up to B needs, hardly more than the largest, and grows with B."""
    plan = getattr(fb.lib(), "_ZN7fluxbin7w4_planERK16fluxbin_w4_shapeii")
    rng = random.Random(2)
    shapes = [(11008, 4096, 64), (512, 28672, 128), (8192, 8192, 32), (100, 20000, 128)]
    shapes += [(int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(6, 17)), rng.choice([32, 64, 128])) for _ in range(60)]
    for M, N, g in shapes:
        s = fb.W4Shape(M, N, g, 0, 0)
        most, before = 0, 0
        for B in range(1, 1200):
            most = max(most, plan(ctypes.addressof(s), B, CUS).ws_bytes)
            n = _workspace()(ctypes.addressof(s), B, CUS)
            assert n >= most and n >= before and (n <= 2 * most + 255 or most == 0 and n == 0), (M, N, g, B)
            before = n


def test_workspace_query_is_quick(form):
    """A call without a workspace asks for its size: not a plan for each smaller batch (0.4 ms of 8192 rows)."""
    import time
    f, s = _workspace(), fb.W4Shape(11008, 4096, 64, 1, 0)
    best = 1.0
    for _ in range(50):
        t = time.perf_counter()
        f(ctypes.addressof(s), 8192, CUS)
        best = min(best, time.perf_counter() - t)
    assert best < 0.15e-3, best
