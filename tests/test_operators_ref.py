"""The float64 restatements behind the operators' GPU tests, checked on their own: gradients against central
differences, the iteration against what it does to singular values."""
import numpy as np
import pytest

import operators_ref as ref


def _rand(seed, *shape):
    return np.random.RandomState(seed).standard_normal(shape)


@pytest.mark.parametrize("gate_kind", ["none", "vector", "rows"])
def test_block_norm_gradient_against_differences(gate_kind):
    rows, F, s, eps = 3, 5, 0.7, 1e-3
    x, y, w1, w2 = _rand(1, rows, F), _rand(2, rows, F), 1 + 0.3 * _rand(3, F), 1 + 0.3 * _rand(4, F)
    gate = dict(none=None, vector=_rand(5, F), rows=_rand(6, rows, F))[gate_kind]
    cx, ch = _rand(7, rows, F), _rand(8, rows, F)            # cotangents of x_out and h

    def value(x, y, w1, w2, gate):
        xo, h = ref.block_norm(x, y, gate, w1, w2, s, eps)
        return (cx * xo).sum() + (ch * h).sum()

    xo, _ = ref.block_norm(x, y, gate, w1, w2, s, eps)
    got = ref.block_norm_backward(xo, y, gate, w1, w2, s, eps, cx, ch)
    args = dict(x=x, y=y, w1=w1, w2=w2, gate=gate)
    for arg, name in (("x", "dx"), ("y", "dy"), ("w1", "dw_pre"), ("w2", "dw_post"), ("gate", "dgate")):
        if args[arg] is None:
            continue
        for at in np.ndindex(args[arg].shape):
            d = 1e-5
            hi, lo = (dict(args, **{arg: args[arg].copy()}) for _ in range(2))
            hi[arg][at] += d
            lo[arg][at] -= d
            diff = (value(**hi) - value(**lo)) / (2 * d)
            assert abs(diff - got[name][at]) <= 1e-7 * max(1.0, abs(diff)), (name, at)


def test_table_gradient_against_differences():
    V, F, s = 4, 3, 1.7
    tokens = np.array([2, -1, 0, 2, 2, 9])
    table, c = _rand(1, V, F), _rand(2, len(tokens), F)
    g = ref.table_grad(c, tokens, V, s)[0]
    for at in np.ndindex(V, F):
        hi, lo = table.copy(), table.copy()
        hi[at] += 0.5
        lo[at] -= 0.5
        diff = (c * (ref.lookup(hi, tokens, s) - ref.lookup(lo, tokens, s))).sum()      # linear: exact
        assert abs(diff - g[at]) < 1e-12


@pytest.mark.parametrize("shape", [(7, 7), (4, 9), (9, 4), (1, 6), (6, 1)])
def test_newton_schulz_moves_singular_values_only(shape):
    G = _rand(3, 1, *shape)
    u, s, vt = np.linalg.svd(G[0], full_matrices=False)
    s = s / np.sqrt((s * s).sum())
    a, b, c = 3.4445, -4.7750, 2.0315
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    np.testing.assert_allclose(ref.newton_schulz(G, 5, (a, b, c), 1e-30)[0], (u * s) @ vt, atol=1e-10)
    cubic = ref.newton_schulz(G, 40, (1.5, -0.5, 0.0), 1e-30)[0]      # converges: U V^T
    np.testing.assert_allclose(cubic, u @ vt, atol=1e-9)
