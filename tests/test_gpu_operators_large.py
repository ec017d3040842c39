"""Lookup, table gradient and norms at row counts that take more than one round, tile or chunk of the kernels."""
import numpy as np
import pytest

import operators_ref as ref
from helpers import tiny_graph
from gpu_common import load_graph

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _generator(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(seed, *shape, dtype="f32"):
    import torch
    return torch.randn(*shape, device="cuda", generator=_generator(seed)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _tokens(seed, rows, V, kind):
    """"thirds": one token holds a third of the rows, in runs and scattered, the rest is spread, one row in 50 has none."""
    import torch
    u = torch.rand(rows, device="cuda", generator=_generator(seed))
    t = (u * V).to(torch.int32).clamp_(max=V - 1)
    if kind == "skewed":
        t = (torch.exp(u * np.log(V + 1.0)) - 1.0).to(torch.int32).clamp_(0, V - 1)
    elif kind == "thirds":
        v = torch.rand(rows, device="cuda", generator=_generator(seed + 1))
        t[v < 0.25] = V // 2
        t[rows // 4:rows // 4 + rows // 12] = V // 2
        t[v > 0.98] = -1
    return t


@pytest.mark.parametrize("rows,V,F", [(98_305, 700, 8), (120_000, 40, 24), (400_000, 5000, 7), (400_000, 1_500_000, 4), (2_000_000, 29_001, 8),
                                      (2_000_003, 3, 16), (1_000_000, 100, 64)])
@pytest.mark.parametrize("kind", ["even", "skewed", "thirds"])
@pytest.mark.parametrize("gd,od", [("f32", "f32"), ("bf16", "bf16")])
def test_gradient(graph, rows, V, F, kind, gd, od):
    import torch
    tok, dout = _tokens(1, rows, V, kind), _normal(2, rows, F, dtype=gd)
    out_dtype = torch.bfloat16 if od == "bf16" else torch.float32
    got = graph.embedding_grad(graph.embedding_plan(tok, V, F), dout, scale=0.5, out_dtype=out_dtype)
    assert torch.equal(got, graph.embedding_grad(graph.embedding_plan(tok, V, F), dout, scale=0.5, out_dtype=out_dtype))
    at = torch.where(tok < 0, V, tok).long()
    want, mag = (torch.zeros(V + 1, F, dtype=torch.float64, device="cuda").index_add_(0, at, t)[:V] for t in (dout.double(), dout.double().abs()))
    cnt = torch.zeros(V + 1, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones(rows, dtype=torch.float64, device="cuda"))[:V]
    # n float32 additions in any order and a product that is exact: n 2^-24 of the sum of magnitudes; a bfloat16 result adds half
    # a unit in its last place
    bound = (cnt[:, None] + 1) * U * 0.5 * mag * 1.001 + (2.0 ** -8 * 0.5 * want.abs() if od == "bf16" else 0)
    assert bool(((got.double() - 0.5 * want).abs() <= bound).all())
    assert bool((got[cnt == 0] == 0).all())


@pytest.mark.parametrize("rows,V,F", [(40_001, 77, 64), (40_001, 300, 256), (100_003, 50, 96), (50_000, 20, 4), (37_889, 9, 513)])
@pytest.mark.parametrize("td,od", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_lookup_is_exact(graph, rows, V, F, td, od):
    import torch
    table, tok = _normal(3, V, F, dtype=td), _tokens(4, rows, V, "thirds")
    out_dtype = torch.bfloat16 if od == "bf16" else torch.float32
    got = graph.embedding_lookup(table, tok, scale=1.7, out_dtype=out_dtype)
    want = torch.where((tok >= 0)[:, None], table.float()[tok.clamp(min=0).long()] * np.float32(1.7).item(), 0.0)     # one float32 product
    assert torch.equal(got, want.to(out_dtype))


@pytest.mark.parametrize("rows,F,dtype,gate_kind", [(200_000, 36, "f32", "rows"), (200_000, 36, "bf16", "vector"), (60_000, 256, "f32", "vector"),
                                                    (90_001, 130, "bf16", "rows"), (40_000, 99, "f32", "none"), (20_000, 1030, "f32", "rows")])
def test_norms(graph, rows, F, dtype, gate_kind):
    """More rows than the grid covers at once, forward and backward, against float64.  25 roundings of a row's sum of squares, half of
    them through the root, and fewer than 8 more per element: 32 units of 2^-24 of the terms added; bfloat16 storage adds 2^-9."""
    s, eps = 0.6, 1e-6
    x, y = _normal(1, rows, F, dtype=dtype), _normal(2, rows, F, dtype=dtype)
    w1, w2 = 1 + 0.2 * _normal(3, F), 1 + 0.2 * _normal(4, F)
    gate = dict(none=lambda: None, vector=lambda: _normal(5, F), rows=lambda: _normal(5, rows, F, dtype=dtype))[gate_kind]()
    host = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    xn, yn, gn, w1n, w2n = (host(t) for t in (x, y, gate, w1, w2))
    xo, h = graph.block_norm(x, w1, y=y, w_post=w2, gate=gate, scale=s, eps=eps)
    xo_ref, h_ref = ref.block_norm(xn, yn, gn, w1n, w2n, s, eps)
    stored = 2.0 ** -8 if dtype == "bf16" else 0.0

    def close(got, want, size):
        assert np.all(np.abs(host(got) - want) <= 32 * U * size + stored * np.abs(want) + 1e-37)

    size = np.abs(xn) + np.abs(xo_ref - xn)
    close(xo, xo_ref, size)
    close(h, h_ref, np.abs(h_ref) + np.abs(h_ref) / np.maximum(np.abs(xo_ref), 1e-30) * size)
    dh = _normal(6, rows, F, dtype=dtype)
    got = graph.block_norm_backward(xo, dh, w1, y=y, w_post=w2, gate=gate, scale=s, eps=eps)
    xs, dhn = host(xo), host(dh)
    want = ref.block_norm_backward(xs, yn, gn, w1n, w2n, s, eps, None, dhn)
    r = 1 / np.sqrt((xs ** 2).mean(1, keepdims=True) + eps)
    a, xh = np.abs(dhn * w1n), np.abs(xs * r)
    D = r * (a + xh * (a * xh).mean(1, keepdims=True))
    close(got["dx"], want["dx"], D)
    ry = 1 / np.sqrt((yn ** 2).mean(1, keepdims=True) + eps)
    yh, b = np.abs(yn * ry), np.abs(s * (1.0 if gn is None else gn) * w2n) * D
    close(got["dy"], want["dy"], 2 * ry * (b + yh * (b * yh).mean(1, keepdims=True)))
    if gate_kind == "rows":
        close(got["dgate"], want["dgate"], 2 * np.abs(s * w2n) * D * yh)
    # sums over rows: 64 units of every term, then at most `rows` additions
    terms = [("dw_pre", np.abs(dhn) * xh), ("dw_post", np.abs(s * (1.0 if gn is None else gn)) * D * yh)]
    if gate_kind == "vector":
        terms.append(("dgate", np.abs(s * w2n) * D * yh))
    for name, term in terms:
        assert np.all(np.abs(host(got[name]) - want[name]) <= (rows + 128) * U * term.sum(0) + 1e-37), name
