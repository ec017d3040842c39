"""Which coefficients of the Newton-Schulz polynomial are accepted: those that keep every singular value in [0, 1] within 2.
Asked of the library without a GPU: for sizes that need a work area, refused coefficients give INVALID_ARGUMENT and accepted
ones, with no work area, WORKSPACE_TOO_SMALL."""
import ctypes

import numpy as np
import pytest

import paper_2511_09261_b200 as gnnco


def _accepted(a, b, c, steps):
    lib = gnnco.load_library()
    handle = ctypes.create_string_buffer(1 << 16)            # nothing of it is read before the answer
    at = ctypes.c_void_p((ctypes.addressof(ctypes.create_string_buffer(1 << 10)) + 255) & ~255)
    p = gnnco.MuonParams(0.0, 0.0, 0.0, 0, steps, a, b, c, 1e-7, None)
    rc = lib.gnnco_orthogonalise(ctypes.cast(handle, ctypes.c_void_p), gnnco.F32, gnnco.F32, 1, 300, 300, at, at, ctypes.byref(p), at, 0,
                                 None)
    assert rc in (gnnco.INVALID_ARGUMENT, gnnco.WORKSPACE_TOO_SMALL)
    return rc == gnnco.WORKSPACE_TOO_SMALL


def _reach(a, b, c, steps):
    """Largest magnitude that singular values in [0, 1] reach, over a fine grid."""
    a, b, c = (float(np.float32(v)) for v in (a, b, c))
    top = most = 1.0
    for _ in range(steps):
        s = np.linspace(0.0, top, 100_001)
        reach = float(np.abs(s * (a + s * s * (b + s * s * c))).max())
        most = max(most, reach)
        if reach > 4.0:
            break
        top = max(top, reach)
    return most


@pytest.mark.parametrize("a,b,c,steps", [(3.4445, -4.7750, 2.0315, 5), (1.5, -0.5, 0.0, 32), (2.0, -1.5, 0.5, 32), (0.5, 0.25, -0.125, 3),
                                         (1.5, -0.5, 1e-18, 10), (1.5, -0.5, -1e-30, 10)])
def test_usual_coefficients(a, b, c, steps):
    assert _reach(a, b, c, steps) < 2 and _accepted(a, b, c, steps)


@pytest.mark.parametrize("a,b,c", [(5.9, -5.0, 0.0), (5.9, -5.0, 1e-18), (5.9, -5.0, -1e-18), (5.9, -5.0, 1e-30), (-5.9, 5.0, 1e-25),
                                   (9.0, 1.0, 1.0), (float("nan"), 0.0, 0.0), (1.0, float("inf"), 0.0)])
def test_coefficients_that_lead_past_two(a, b, c):
    assert not _accepted(a, b, c, 5)


def test_against_a_grid():
    rng = np.random.RandomState(1)
    seen = {True: 0, False: 0}
    for _ in range(400):
        a, b = rng.uniform(-4, 6), rng.uniform(-6, 4)
        c = rng.choice([-1.0, 1.0]) * 10.0 ** rng.uniform(-40, 0.7)
        steps = int(rng.randint(1, 4))
        reach = _reach(a, b, c, steps)
        if abs(reach - 2.0) < 1e-4:
            continue                                        # nearer than the grid can tell
        assert _accepted(a, b, c, steps) == (reach < 2.0), (a, b, c, steps, reach)
        seen[reach < 2.0] += 1
    assert min(seen.values()) > 40
