"""Shared input embeddings on the GPU: lookup, order by token, table gradient, against the float64 restatement."""
import numpy as np
import pytest

import operators_ref as ref
from helpers import tiny_graph
from gpu_common import load_graph, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _torch_dtype(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _data(seed, rows, F, dtype):
    import torch
    x = np.random.RandomState(seed).standard_normal((rows, F)).astype(np.float32)
    t = torch.from_numpy(x).to(_torch_dtype(dtype))
    return t.cuda(), t.float().numpy()


def _tokens(seed, rows, V, kind):
    r = np.random.RandomState(seed)
    if kind == "one":
        t = np.full(rows, V - 1)
    elif kind == "none":
        t = np.full(rows, -1)
    elif kind == "skewed":
        t = np.floor(V ** r.rand(rows) - 1).clip(0, V - 1)
    else:
        t = r.randint(-1, V, rows)
    return t.astype(np.int32)


@pytest.mark.parametrize("td,od", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,V,F", [(1, 1, 1), (5, 3, 7), (257, 40, 64), (1000, 33, 100), (4099, 301, 256), (40_001, 77, 24),
                                      (31, 5, 2050)])
def test_lookup_is_exact(graph, td, od, rows, V, F):
    import torch
    table, host = _data(1, V, F, td)
    tok = _tokens(2, rows, V, "mixed")
    got = graph.embedding_lookup(table, to_dev(tok), scale=1.7, out_dtype=_torch_dtype(od))
    want = np.where((tok >= 0)[:, None], host[tok.clip(0)] * np.float32(1.7), np.float32(0))       # one float32 product
    assert got.dtype == _torch_dtype(od)
    assert torch.equal(got.cpu(), torch.from_numpy(want).to(_torch_dtype(od)))


@pytest.mark.parametrize("off,wide", [(0, 300), (8, 304), (3, 301), (4, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lookup_and_gradient_on_columns_of_wider_tensors(graph, dtype, off, wide):
    import torch
    rows, V, F = 700, 19, 96
    big_table, host = _data(3, V, wide, dtype)
    tok = _tokens(4, rows, V, "skewed")
    out = torch.full((rows, wide), 7.0, dtype=_torch_dtype(dtype), device="cuda")
    graph.embedding_lookup(big_table[:, off:off + F], to_dev(tok), scale=0.5, out=out[:, off:off + F])
    want = torch.full((rows, wide), 7.0)
    want[:, off:off + F] = torch.from_numpy(host[tok, off:off + F] * np.float32(0.5))
    assert torch.equal(out.cpu(), want.to(_torch_dtype(dtype)))
    plan = graph.embedding_plan(to_dev(tok), V, F)
    dense = graph.embedding_grad(plan, out[:, off:off + F].contiguous(), scale=2.0)
    g = torch.full((V, wide), 7.0, device="cuda")
    graph.embedding_grad(plan, out[:, off:off + F], scale=2.0, out=g[:, off:off + F])
    assert torch.equal(g[:, off:off + F], dense)
    g[:, off:off + F] = 7.0
    assert bool((g == 7.0).all())


@pytest.mark.parametrize("kind", ["mixed", "skewed", "one", "none"])
@pytest.mark.parametrize("gd,od", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,V,F", [(1, 1, 1), (3, 700, 5), (15, 4, 64), (16, 4, 64), (17, 4, 64), (1000, 33, 100), (4096, 257, 72),
                                      (4097, 256, 40), (20_000, 70_001, 16), (60_000, 513, 33)])
def test_gradient(graph, rows, V, F, gd, od, kind):
    import torch
    dout, host = _data(5, rows, F, gd)
    tok = _tokens(6, rows, V, kind)
    plan = graph.embedding_plan(to_dev(tok), V, F)
    got = graph.embedding_grad(plan, dout, scale=-0.75, out_dtype=_torch_dtype(od))
    again = graph.embedding_grad(graph.embedding_plan(to_dev(tok), V, F), dout, scale=-0.75, out_dtype=_torch_dtype(od))
    assert torch.equal(got, again)                                     # the order of every sum is fixed
    want, mag, cnt = ref.table_grad(host, tok, V, -0.75)
    # n float32 additions in any order: at most n 2^-24 of the sum of magnitudes, plus the product with the scale; a
    # bfloat16 result adds half a unit in its last place
    bound = (cnt[:, None] + 1) * 2.0 ** -24 * mag * 1.001 + (2.0 ** -8 * np.abs(want) if od == "bf16" else 0)
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound)
    assert np.all(got.float().cpu().numpy()[cnt == 0] == 0)


def test_gradient_of_a_narrower_table_from_one_plan(graph):
    import torch
    tok = to_dev(_tokens(7, 5000, 90, "skewed"))
    plan = graph.embedding_plan(tok, 90, 128)
    for F in (128, 31, 4):
        dout, _ = _data(8, 5000, F, "f32")
        assert torch.equal(graph.embedding_grad(plan, dout), graph.embedding_grad(graph.embedding_plan(tok, 90, F), dout))


def test_no_rows(graph):
    import torch
    tok = torch.empty(0, dtype=torch.int32, device="cuda")
    table, _ = _data(1, 5, 8, "f32")
    assert graph.embedding_lookup(table, tok).shape == (0, 8)
    g = graph.embedding_grad(graph.embedding_plan(tok, 5, 8), torch.empty(0, 8, device="cuda"), out=torch.ones(5, 8, device="cuda"))
    assert not g.any()


@pytest.mark.parametrize("rows", [50, 9000])
def test_tokens_past_the_table_are_reported_and_skipped(rows):
    import torch
    import paper_2511_09261_b200 as gnnco
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    for use in ("lookup", "plan"):
        g = load_graph(64, eu, ev, part, int(part.max()) + 1)
        tok = _tokens(3, rows, 7, "mixed")
        tok[rows // 2] = 7
        if use == "lookup":
            table, host = _data(1, 7, 8, "f32")
            out = g.embedding_lookup(table, to_dev(tok))
            assert not out[rows // 2].any()
        else:
            dout, host = _data(2, rows, 8, "f32")
            want, mag, cnt = ref.table_grad(host, tok, 7, 1.0)
            got = g.embedding_grad(g.embedding_plan(to_dev(tok), 7, 8), dout).double().cpu().numpy()
            assert np.all(np.abs(got - want) <= (cnt[:, None] + 1) * 2.0 ** -24 * mag * 1.001)
        assert g.async_status() == gnnco.OUT_OF_RANGE


def test_infinities_and_nans_stay_in_their_row(graph):
    import torch
    tok = to_dev(np.array([0, 1, 2, 1, -1], np.int32))
    dout = torch.ones(5, 8, device="cuda")
    dout[1, 3], dout[2, 4], dout[4] = float("inf"), float("nan"), float("nan")
    g = graph.embedding_grad(graph.embedding_plan(tok, 4, 8), dout).cpu()
    want = torch.tensor([1.0, 2.0, 1.0, 0.0])[:, None].repeat(1, 8)
    want[1, 3], want[2, 4] = float("inf"), float("nan")
    assert torch.equal(torch.nan_to_num(g, nan=-5.0), torch.nan_to_num(want, nan=-5.0))


def test_on_another_stream(graph):
    import torch
    table, host = _data(1, 50, 64, "f32")
    tok = to_dev(_tokens(2, 3000, 50, "mixed"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = graph.embedding_lookup(table, tok, stream=side)
    g = graph.embedding_grad(graph.embedding_plan(tok, 50, 64, stream=side), out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, graph.embedding_lookup(table, tok))
    assert torch.equal(g, graph.embedding_grad(graph.embedding_plan(tok, 50, 64), out))


def test_refusals(graph):
    import ctypes
    import torch
    import paper_2511_09261_b200 as gnnco
    table, _ = _data(1, 5, 8, "f32")
    tok = to_dev(np.zeros(4, np.int32))
    for bad in (dict(table=table.half()), dict(tokens=tok.long()), dict(tokens=tok.cpu()), dict(table=table.cpu()),
                dict(out_dtype=torch.float16)):
        with pytest.raises(TypeError):
            graph.embedding_lookup(**{**dict(table=table, tokens=tok), **bad})
    for bad in (dict(table=table.t()), dict(tokens=tok.view(2, 2)), dict(out=torch.empty(4, 9, device="cuda")),
                dict(out=torch.empty(1, 8, device="cuda").expand(4, 8))):
        with pytest.raises(ValueError):
            graph.embedding_lookup(**{**dict(table=table, tokens=tok), **bad})
    plan = graph.embedding_plan(tok, 5, 8)
    with pytest.raises(ValueError):
        graph.embedding_grad(plan, torch.empty(4, 9, device="cuda"))
    with pytest.raises(ValueError):
        graph.embedding_grad(plan, torch.empty(3, 8, device="cuda"))
    with pytest.raises(gnnco.GnncoError):
        graph.embedding_plan(tok, 0, 8)
    lib, h = gnnco.load_library(), graph._handle
    assert lib.gnnco_embedding_plan(h, tok.data_ptr(), 4, 5, 8, plan.ws.data_ptr(), 256, None) == gnnco.WORKSPACE_TOO_SMALL
    assert lib.gnnco_embedding_plan(h, tok.data_ptr(), 4, 5, 8, plan.ws.data_ptr() + 16, 1 << 20, None) == gnnco.INVALID_ARGUMENT
    args = (table.data_ptr(), 8, 1.0, table.data_ptr(), 8, None)
    assert lib.gnnco_embedding_lookup(None, 0, 0, 4, 5, 8, tok.data_ptr(), *args) == gnnco.INVALID_ARGUMENT
    assert lib.gnnco_embedding_lookup(h, 2, 0, 4, 5, 8, tok.data_ptr(), *args) == gnnco.UNSUPPORTED
    assert lib.gnnco_embedding_lookup(h, 0, 0, -1, 5, 8, tok.data_ptr(), *args) == gnnco.INVALID_ARGUMENT
    assert lib.gnnco_embedding_lookup(h, 0, 0, 4, 5, 9, tok.data_ptr(), *args) == gnnco.INVALID_ARGUMENT
