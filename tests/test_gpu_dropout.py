"""Dropout on the GPU against the float64 restatement: which elements stay is compared exactly, their values to the rounding of
one product and one conversion."""
import numpy as np
import pytest

import ff_ref as ref
from helpers import tiny_graph
from gpu_common import load_graph

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _x(rows, F, dtype, seed=1):
    import torch
    t = torch.from_numpy(np.random.RandomState(seed).standard_normal((rows, F)).astype(np.float32) + 3.0)
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def _check(got, x, p, **at):
    """The factor 1 / (1 - p) is rounded to float32, the product once more (2 x 2^-24), and the result to its type (bfloat16 2^-8)."""
    want = ref.dropout(x.float().cpu().numpy(), p, **at)
    got = got.double().cpu().numpy()
    assert np.array_equal(got == 0.0, want == 0.0)
    bound = (2.0 ** -23 * (1 + 2.0 ** -20) + (2.0 ** -8 if x.element_size() == 2 else 0.0)) * np.abs(want)
    assert np.all(np.abs(got - want) <= bound)


SHAPES = [(1, 1), (1, 4), (2, 3), (5, 7), (1, 8), (3, 12), (33, 8), (130, 99), (257, 64), (1000, 4), (31, 1000), (2, 5001), (4099, 20)]


@pytest.mark.parametrize("rows,F", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_values_and_mask(graph, rows, F, dtype, p):
    import paper_2511_09261_b200 as gnnco
    x = _x(rows, F, dtype)
    _check(graph.dropout(x, gnnco.Dropout(p, 0x123456789ABCDEF0, layer=7, step=11)), x, p, seed=0x123456789ABCDEF0, layer=7, step=11)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,offset", [(24, 0), (24, 8), (25, 1), (30, 2), (28, 4)])
def test_columns_of_wider_tensors(graph, dtype, ld, offset):
    import torch
    x, out = _x(300, ld, dtype), _x(300, ld, dtype, 2)
    before = out.clone()
    cols = slice(offset, offset + 16)
    graph.dropout(x[:, cols], gnnco_drop(0.3), out=out[:, cols])
    _check(out[:, cols], x[:, cols], 0.3, seed=42)
    out[:, cols] = before[:, cols]
    assert torch.equal(out, before)


def gnnco_drop(p, **k):
    import paper_2511_09261_b200 as gnnco
    return gnnco.Dropout(p, 42, **k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [8, 7])
def test_all_none_empty_and_in_place(graph, dtype, F):
    import torch
    x = _x(100, F, dtype)
    assert torch.equal(graph.dropout(x, gnnco_drop(0.0)), x)
    assert torch.equal(graph.dropout(x, gnnco_drop(1e-11)), x)              # below 2^-33: nothing is dropped
    assert not graph.dropout(x, gnnco_drop(1.0)).any()
    assert graph.dropout(x[:0], gnnco_drop(0.5)).shape == (0, F)
    want = graph.dropout(x, gnnco_drop(0.5))
    assert graph.dropout(x, gnnco_drop(0.5), out=x) is x and torch.equal(x, want)


@pytest.mark.parametrize("F", [8, 5])
def test_dropped_infinities_and_nans_are_gone(graph, F):
    import torch
    x = torch.full((64, F), float("nan"), device="cuda")
    x[::2] = float("inf")
    on = ref.keep(64, F, 0.5, 42)
    got = graph.dropout(x, gnnco_drop(0.5)).cpu().numpy()
    assert np.array_equal(got == 0.0, ~on)
    assert np.array_equal(np.isnan(got), on & np.isnan(x.cpu().numpy()))


def test_quads_past_32_bits_and_rows_past_a_round_of_the_grid(graph):
    """2^32 quads take 32 GB in bfloat16; the last rows are the ones whose counter has a second word."""
    import torch
    rows, F = (1 << 24) + 5, 1024
    x = torch.ones(rows, F, dtype=torch.bfloat16, device="cuda")
    graph.dropout(x, gnnco_drop(0.5), out=x)
    for row0 in (0, 1 << 20, (1 << 24) - 3):
        got = x[row0:row0 + 8].cpu().float().numpy()
        assert np.array_equal(got != 0.0, ref.keep(8, F, 0.5, 42, row0=row0)), row0


def test_gradient_is_the_same_call(graph):
    """out is linear in x: <out(x), dy> = <x, out(dy)> term by term, with the same elements kept."""
    x, dy = _x(50, 30, "f32"), _x(50, 30, "f32", 3)
    a, b = graph.dropout(x, gnnco_drop(0.4)), graph.dropout(dy, gnnco_drop(0.4))
    assert np.array_equal((a != 0).cpu().numpy(), (b != 0).cpu().numpy())
    left, right = (a.double() * dy.double()).sum().item(), (x.double() * b.double()).sum().item()
    assert abs(left - right) <= 2.0 ** -22 * (a.double() * dy.double()).abs().sum().item()


def test_a_recorded_graph_draws_new_masks_as_the_step_advances(graph):
    import torch
    x = _x(200, 32, "f32")
    step = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    drop = gnnco_drop(0.5, layer=2, step=100, step_dev=step)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph.dropout(x, drop)
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        out = graph.dropout(x, drop)
        step.add_(1)
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        _check(out, x, 0.5, seed=42, layer=2, step=105 + k)


def test_another_stream(graph):
    import torch
    x = _x(5000, 64, "bf16")
    want = graph.dropout(x, gnnco_drop(0.2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = graph.dropout(x, gnnco_drop(0.2), stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("p", [0.0, 0.5])
def test_rows_far_apart(graph, p):
    """Two rows 2^30 elements (4 GB) apart, more than a strided copy takes as its pitch."""
    import torch
    import paper_2511_09261_b200 as gnnco
    base = torch.empty((1 << 30) + 5, dtype=torch.float32, device="cuda")
    x = base.as_strided((2, 5), (1 << 30, 1))
    x.copy_(torch.arange(1.0, 11.0).view(2, 5))
    drop = gnnco.Dropout(p, 7)
    want = graph.dropout(x.clone(memory_format=torch.contiguous_format), drop)
    assert torch.equal(graph.dropout(x, drop), want)
    assert torch.equal(graph.dropout(x, drop, out=x), want)
    if p == 0.0:
        out = torch.zeros(2, 7, device="cuda")
        graph.dropout(x, drop, out=out[:, :5])
        assert torch.equal(out[:, :5], want) and not out[:, 5:].any()
