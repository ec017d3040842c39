"""Norms around a block with gate and residual scale on the GPU, forward and backward, against the float64 restatement."""
import numpy as np
import pytest

import operators_ref as ref
from helpers import tiny_graph
from gpu_common import load_graph, to_dev

pytestmark = pytest.mark.gpu
EPS = 1e-6
U = 2.0 ** -24


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _feat(seed, rows, F, dtype, scale=1.0, mean=0.0):
    import torch
    x = (mean + scale * np.random.RandomState(seed).standard_normal((rows, F))).astype(np.float32)
    t = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t.cuda(), t.float().numpy()


def _vec(seed, F):
    return (1.0 + 0.2 * np.random.RandomState(seed).standard_normal(F)).astype(np.float32)


def _close(got, want, dtype, scale_rows):
    """A row's statistics are sums of F terms of one sign, each lane adding at most 16 before a tree of at most 9 levels:
    25 roundings, half of them through the square root, and fewer than 8 more per element: 32 units of 2^-24 on every term.
    `scale_rows` is the size of the terms that were added (they may cancel); bfloat16 storage adds half a unit in the last
    place, 2^-9 relative."""
    got = got.double().cpu().numpy()
    bound = 32 * U * scale_rows + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-37
    assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())


def _case(rows, F, dtype, gate_kind, weights):
    x, xn = _feat(1, rows, F, dtype)
    y, yn = _feat(2, rows, F, dtype, 3.0, 0.5)
    gate = gn = None
    if gate_kind == "vector":
        gn = _vec(3, F)
        gate = to_dev(gn)
    elif gate_kind == "rows":
        gate, gn = _feat(4, rows, F, dtype, 0.4, 0.3)
    w1, w2 = (_vec(5, F), _vec(6, F)) if weights else (None, None)
    dev = lambda w: None if w is None else to_dev(w)  # noqa: E731
    return (x, y, gate, dev(w1), dev(w2)), (xn, yn, gn, w1, w2)


SHAPES = [(1, 1), (3, 2), (5, 8), (7, 64), (130, 99), (33, 100), (65, 128), (40, 250), (300, 256), (9, 257), (17, 512), (11, 520),
          (6, 1000), (5, 1024), (4, 2048), (3, 2049), (3, 4096), (2, 8191), (2, 8192)]


@pytest.mark.parametrize("rows,F", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate_kind,weights", [("none", False), ("vector", True), ("rows", True)])
def test_forward_and_backward(graph, rows, F, dtype, gate_kind, weights):
    s = 0.6
    (x, y, gate, w1, w2), (xn, yn, gn, w1n, w2n) = _case(rows, F, dtype, gate_kind, weights)
    xo, h = graph.block_norm(x, w1, y=y, w_post=w2, gate=gate, scale=s, eps=EPS)
    xo_ref, h_ref = ref.block_norm(xn, yn, gn, w1n, w2n, s, EPS)
    block = np.abs(xo_ref - xn)
    _close(xo, xo_ref, dtype, np.abs(xn) + block)
    gain = np.abs(h_ref) / np.maximum(np.abs(xo_ref), 1e-30)
    _close(h, h_ref, dtype, np.abs(h_ref) + gain * (np.abs(xn) + block))

    xo_in = xo.float().cpu().numpy()
    dx_out, dxn = _feat(7, rows, F, dtype)
    dh, dhn = _feat(8, rows, F, dtype)
    got = graph.block_norm_backward(xo, dh, w1, dx_out=dx_out, y=y, w_post=w2, gate=gate, scale=s, eps=EPS)
    want = ref.block_norm_backward(xo_in, yn, gn, w1n, w2n, s, EPS, dxn, dhn)
    # sizes of the terms behind dx and dy (both are differences), with the means taken over magnitudes
    r = 1 / np.sqrt((xo_in.astype(np.float64) ** 2).mean(1, keepdims=True) + EPS)
    a = np.abs(dhn * (1.0 if w1n is None else w1n))
    xh = np.abs(xo_in * r)
    D_size = np.abs(dxn) + r * (a + xh * (a * xh).mean(1, keepdims=True))
    _close(got["dx"], want["dx"], dtype, D_size)
    ry = 1 / np.sqrt((yn.astype(np.float64) ** 2).mean(1, keepdims=True) + EPS)
    yh = np.abs(yn * ry)
    g = np.abs(s * (1.0 if gn is None else gn) * (1.0 if w2n is None else w2n))
    b = g * D_size
    _close(got["dy"], want["dy"], dtype, 2 * ry * (b + yh * (b * yh).mean(1, keepdims=True)))
    # sums over rows: every term carries the errors above (64 units of the term's own size), then at most rows + 64 additions
    if weights:
        for name, term in (("dw_pre", np.abs(dhn) * xh), ("dw_post", np.abs(s * gn) * D_size * yh)):
            bound = (rows + 128) * U * term.sum(0) + 1e-37
            assert np.all(np.abs(got[name].double().cpu().numpy() - want[name]) <= bound), name
    if gate_kind == "vector":
        bound = (rows + 128) * U * (np.abs(s * w2n) * D_size * yh).sum(0) + 1e-37
        assert np.all(np.abs(got["dgate"].double().cpu().numpy() - want["dgate"]) <= bound)
    elif gate_kind == "rows":
        _close(got["dgate"], want["dgate"], dtype, 2 * np.abs(s * w2n) * D_size * yh)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_that_may_be_left_out(graph, dtype):
    import torch
    rows, F = 77, 72
    (x, y, gate, w1, w2), (xn, yn, gn, w1n, w2n) = _case(rows, F, dtype, "vector", True)
    # before the first block: only a norm
    same, h = graph.block_norm(x, w1, eps=EPS)
    assert same is x
    _, h_ref = ref.block_norm(xn, None, None, w1n, None, 1.0, EPS)
    _close(h, h_ref, dtype, 2 * np.abs(h_ref))
    # after the last block: only the residual
    xo, none = graph.block_norm(x, y=y, w_post=w2, gate=gate, scale=0.6, eps=EPS, want_h=False)
    assert none is None
    assert torch.equal(xo, graph.block_norm(x, w1, y=y, w_post=w2, gate=gate, scale=0.6, eps=EPS)[0])
    # their gradients
    dh, dhn = _feat(8, rows, F, dtype)
    got = graph.block_norm_backward(x, dh, w1, eps=EPS)
    assert got["dy"] is None and got["dgate"] is None and got["dw_post"] is None
    zero = torch.zeros_like(dh)
    assert torch.equal(got["dx"], graph.block_norm_backward(x, dh, w1, dx_out=zero, eps=EPS)["dx"])
    got = graph.block_norm_backward(xo, dx_out=dh, y=y, w_post=w2, gate=gate, scale=0.6, eps=EPS)
    assert torch.equal(got["dx"], dh) and got["dw_pre"] is None
    full = graph.block_norm_backward(xo, zero, w1, dx_out=dh, y=y, w_post=w2, gate=gate, scale=0.6, eps=EPS)
    assert torch.equal(got["dy"], full["dy"]) and torch.equal(got["dgate"], full["dgate"])
    assert not full["dw_pre"].any()


@pytest.mark.parametrize("F", [64, 99, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_in_place_and_repeatable(graph, dtype, F):
    import torch
    rows = 211
    (x, y, gate, w1, w2), _ = _case(rows, F, dtype, "rows", True)
    want = graph.block_norm(x, w1, y=y, w_post=w2, gate=gate, scale=0.5, eps=EPS)
    dh, dxo = _feat(8, rows, F, dtype)[0], _feat(9, rows, F, dtype)[0]
    grads = graph.block_norm_backward(want[0], dh, w1, dx_out=dxo, y=y, w_post=w2, gate=gate, scale=0.5, eps=EPS)
    for pad, off in ((16, 8), (5, 3)):
        def wide(t):
            w = torch.full((rows, F + pad), 9.0, dtype=t.dtype, device="cuda")
            w[:, off:off + F] = t
            return w[:, off:off + F]
        xs = wide(x)
        xo, h = graph.block_norm(xs, w1, y=wide(y), w_post=w2, gate=wide(gate), scale=0.5, eps=EPS, x_out=xs, h_out=wide(x))
        assert xo.data_ptr() == xs.data_ptr()
        # another vector width may add a row's squares in another order: the outputs agree to the tests' own bounds
        tol = dict(rtol=2e-5, atol=2e-5) if dtype == "f32" else dict(rtol=2.0 ** -7, atol=1e-4)
        torch.testing.assert_close(xo, want[0], **tol)
        torch.testing.assert_close(h, want[1], **tol)
        d = wide(dxo)
        got = graph.block_norm_backward(wide(want[0]), wide(dh), w1, dx_out=d, y=wide(y), w_post=w2, gate=wide(gate), scale=0.5,
                                        eps=EPS, dx=d, dy=wide(y), dgate=wide(y))
        for name in ("dx", "dy", "dgate"):
            torch.testing.assert_close(got[name], grads[name], **tol)
        base = d._base
        assert bool((base[:, :off] == 9.0).all()) and bool((base[:, off + F:] == 9.0).all())
    again = graph.block_norm_backward(want[0], dh, w1, dx_out=dxo, y=y, w_post=w2, gate=gate, scale=0.5, eps=EPS)
    assert all(torch.equal(again[k], grads[k]) for k in grads)


def test_many_rows_and_weight_sums(graph):
    rows, F = 50_001, 36
    (x, y, gate, w1, w2), (xn, yn, gn, w1n, w2n) = _case(rows, F, "f32", "vector", True)
    dh, dhn = _feat(8, rows, F, "f32")
    got = graph.block_norm_backward(x, dh, w1, y=y, w_post=w2, gate=gate, scale=0.5, eps=EPS)
    want = ref.block_norm_backward(xn, yn, gn, w1n, w2n, 0.5, EPS, None, dhn)
    for name in ("dw_pre", "dw_post", "dgate"):
        # fixed order of at most rows / (blocks x teams) + a few hundred additions: far below rows
        assert np.all(np.abs(got[name].double().cpu().numpy() - want[name]) <= 600 * U * want[name + "_mag"]), name


def test_zero_rows_and_extreme_values(graph):
    import torch
    x = torch.zeros(6, 32, device="cuda")
    x[1], x[2], x[3, 0], x[4, 5] = 1e15, 1e-22, float("inf"), float("nan")
    x[5] = 2.0
    xo, h = graph.block_norm(x, eps=EPS)
    h = h.cpu().numpy()
    assert np.all(h[0] == 0) and np.allclose(h[1], 1.0, rtol=1e-6) and np.allclose(h[2], 1e-22 / np.sqrt(EPS), rtol=1e-5)
    assert np.isnan(h[3, 0]) and np.all(h[3, 1:] == 0) and np.all(np.isnan(h[4])) and np.allclose(h[5], 1.0, rtol=1e-5)
    got = graph.block_norm_backward(x[:3].contiguous(), torch.ones(3, 32, device="cuda"), eps=EPS)["dx"].cpu().numpy()
    assert np.allclose(got[0], 1 / np.sqrt(EPS), rtol=1e-5) and np.all(np.isfinite(got))
    # no rows at all: sums are zero
    e = torch.empty(0, 32, device="cuda")
    w = torch.ones(32, device="cuda")
    assert graph.block_norm(e, w, y=e, w_post=w, gate=w)[1].shape == (0, 32)
    g = graph.block_norm_backward(e, e, w, y=e, w_post=w, gate=w)
    assert not g["dw_pre"].any() and not g["dw_post"].any() and not g["dgate"].any()


def test_gradient_against_differences_on_the_gpu(graph):
    """Directional derivative of <c, h> + <d, x_out> in float32: the difference quotient's error is |step|^2 times third
    derivatives (O(1) here) plus 2^-24 sqrt(values) / step of rounding: 5e-3 at a step of 1e-2 covers both."""
    import torch
    rows, F, s = 64, 48, 0.8
    (x, y, gate, w1, w2), _ = _case(rows, F, "f32", "vector", True)
    c, d, v, vy = (_feat(k, rows, F, "f32")[0] for k in (11, 12, 13, 14))

    def value(x, y):
        xo, h = graph.block_norm(x, w1, y=y, w_post=w2, gate=gate, scale=s, eps=1e-2)
        return float((c.double() * h.double()).sum() + (d.double() * xo.double()).sum())

    xo, _ = graph.block_norm(x, w1, y=y, w_post=w2, gate=gate, scale=s, eps=1e-2)
    g = graph.block_norm_backward(xo, c, w1, dx_out=d, y=y, w_post=w2, gate=gate, scale=s, eps=1e-2)
    e = 1e-2
    slope = (value(x + e * v, y + e * vy) - value(x - e * v, y - e * vy)) / (2 * e)
    want = float((g["dx"].double() * v.double()).sum() + (g["dy"].double() * vy.double()).sum())
    size = float((g["dx"].double() * v.double()).abs().sum() + (g["dy"].double() * vy.double()).abs().sum())
    assert abs(slope - want) <= 5e-3 * np.sqrt(rows * F) + 1e-4 * size


def test_refusals(graph):
    import ctypes
    import torch
    import paper_2511_09261_b200 as gnnco
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda")
    for bad in (dict(x=x.half()), dict(x=x, y=x.bfloat16()), dict(x=x, w_pre=w.bfloat16()), dict(x=x, y=x, gate=x.bfloat16())):
        with pytest.raises(TypeError):
            graph.block_norm(**bad)
    for bad in (dict(x=x, gate=w), dict(x=x, w_post=w), dict(x=x, w_pre=w[:7].contiguous()), dict(x=x, y=x[:3]), dict(x=x.t()[:, :3], y=x),
                dict(x=x, x_out=x)):
        with pytest.raises(ValueError):
            graph.block_norm(**bad)
    for call in (lambda: graph.block_norm(x, eps=0.0), lambda: graph.block_norm(x, want_h=False), lambda: graph.block_norm(x, eps=float("nan")),
                 lambda: graph.block_norm_backward(x)):
        with pytest.raises(gnnco.GnncoError) as e:
            call()
        assert e.value.status == gnnco.INVALID_ARGUMENT
    with pytest.raises(gnnco.GnncoError) as e:
        graph.block_norm(torch.ones(2, 8193, device="cuda"))
    assert e.value.status == gnnco.UNSUPPORTED
    lib, h = gnnco.load_library(), graph._handle
    d = graph._block_desc(x, None, None, None, None, 1.0, EPS)
    g = gnnco.BlockNormGrads(None, 0, x.data_ptr(), 8, x.data_ptr(), 8)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert lib.gnnco_block_norm_backward(h, ctypes.byref(d), ctypes.byref(g), ws.data_ptr(), 256, None) == gnnco.WORKSPACE_TOO_SMALL
    assert lib.gnnco_block_norm_backward(h, ctypes.byref(d), ctypes.byref(g), ws.data_ptr() + 8, 1 << 19, None) == gnnco.INVALID_ARGUMENT
    assert lib.gnnco_block_norm(None, ctypes.byref(d), None, 0, x.data_ptr(), 8, None) == gnnco.INVALID_ARGUMENT
    d.feat_dtype = 5
    assert lib.gnnco_block_norm(h, ctypes.byref(d), None, 0, x.data_ptr(), 8, None) == gnnco.UNSUPPORTED
