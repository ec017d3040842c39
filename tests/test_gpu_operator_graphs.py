"""The operators around a step recorded in CUDA graphs: what a graph keeps is its own."""
import numpy as np
import pytest

from helpers import tiny_graph
from gpu_common import load_graph, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _normal(seed, *shape):
    import torch
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _record(call, stream):
    """A CUDA graph of `call` recorded on `stream`, after one ordinary call there, and what the call returned."""
    import torch
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        out = call()
    return g, out


def _norm_inputs(seed, rows, F):
    return dict(x=_normal(seed, rows, F), dh=_normal(seed + 1, rows, F), w_pre=_normal(seed + 2, F), y=_normal(seed + 3, rows, F),
                w_post=_normal(seed + 4, F), gate=_normal(seed + 5, F))


def test_norm_gradients_of_a_graph_and_of_calls_beside_it(graph):
    """A later call with wider rows on the recording stream, and tensors that are made after it, leave a recorded backward pass
    alone, and its replay leaves them alone."""
    import torch
    small, wide = _norm_inputs(1, 3000, 64), _norm_inputs(11, 3000, 256)
    want, want_wide = graph.block_norm_backward(**small), graph.block_norm_backward(**wide)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph.block_norm_backward(**small, stream=stream)
    g, got = _record(lambda: graph.block_norm_backward(**small, stream=stream), stream)
    got_wide = graph.block_norm_backward(**wide, stream=stream)
    stream.synchronize()
    with torch.cuda.stream(stream):
        fill = [torch.full((1 << 16,), 7.0, device="cuda") for _ in range(200)]
    stream.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    assert all(torch.equal(got_wide[k], want_wide[k]) for k in want)
    assert all(bool((t == 7.0).all()) for t in fill)


def test_two_graphs_recorded_on_one_stream_share_no_work_area(graph):
    """... and may be replayed side by side."""
    import torch
    a, b = _norm_inputs(1, 200_000, 128), _norm_inputs(11, 200_000, 128)
    want = [graph.block_norm_backward(**v) for v in (a, b)]
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    ga, got_a = _record(lambda: graph.block_norm_backward(**a, stream=stream), stream)
    gb, got_b = _record(lambda: graph.block_norm_backward(**b, stream=stream), stream)
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(stream):
            ga.replay()
        with torch.cuda.stream(other):
            gb.replay()
    torch.cuda.synchronize()
    for want_one, got in zip(want, (got_a, got_b)):
        assert all(torch.equal(got[k], want_one[k]) for k in want_one)


def test_a_plan_dropped_while_another_stream_uses_it(graph):
    """The gradient waits on its stream behind other work when the plan goes; memory that is asked for then must not be the plan's."""
    import torch
    rows, V, F = 50_000, 1000, 32
    tokens = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    dout = _normal(2, rows, F)
    want = graph.embedding_grad(graph.embedding_plan(tokens, V, F), dout)
    plan = graph.embedding_plan(tokens, V, F)
    size = plan.ws.shape[0]
    stream = torch.cuda.Stream()
    out, factor = torch.empty_like(want), _normal(3, 4096, 4096)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):
            factor @ factor
    graph.embedding_grad(plan, dout, out=out, stream=stream)
    del plan
    others = [torch.full((size,), 1, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all(bool((t == 1).all()) for t in others)


@pytest.mark.parametrize("rows", [3000, 150_000])
def test_lookup_order_and_gradient_replay_on_new_inputs(graph, rows):
    import torch
    V, F = 500, 40
    make = lambda seed: torch.randint(-1, V, (rows,), device="cuda", dtype=torch.int32,  # noqa: E731
                                      generator=torch.Generator(device="cuda").manual_seed(seed))
    table, tokens, dout = _normal(1, V, F), make(1), _normal(2, rows, F)
    stream = torch.cuda.Stream()

    def call():
        return (graph.embedding_lookup(table, tokens, scale=2.0, stream=stream),
                graph.embedding_grad(graph.embedding_plan(tokens, V, F, stream=stream), dout, scale=2.0, stream=stream))

    g, got = _record(call, stream)
    for seed in (3, 4):
        table.copy_(_normal(seed, V, F))
        tokens.copy_(make(seed))
        dout.copy_(_normal(seed + 10, rows, F))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], graph.embedding_lookup(table, tokens, scale=2.0))
        assert torch.equal(got[1], graph.embedding_grad(graph.embedding_plan(tokens, V, F), dout, scale=2.0))


@pytest.mark.parametrize("sets,r,c", [(300, 16, 9), (400, 64, 32), (60, 100, 200), (100, 200, 140), (3, 300, 400), (1, 70, 2700)])
def test_updates_replay_on_new_inputs(graph, sets, r, c):
    import torch
    W, m, d = _normal(1, sets, r, c), _normal(2, sets, r, c), _normal(3, sets, r, c)
    W2, m2 = W.clone(), m.clone()
    stream = torch.cuda.Stream()
    g, _ = _record(lambda: graph.muon_update(W, m, d, lr=0.1, weight_decay=0.1, stream=stream), stream)
    W.copy_(W2)
    m.copy_(m2)
    for seed in (5, 6, 7):
        d.copy_(_normal(seed, sets, r, c))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        graph.muon_update(W2, m2, d, lr=0.1, weight_decay=0.1)
        assert torch.equal(W, W2) and torch.equal(m, m2)
    assert graph.async_status() == 0
