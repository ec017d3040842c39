"""What the binding of the operators around a step keeps and checks, without a GPU: the library behind it is a stand-in that
records its arguments."""
import ctypes

import pytest
import torch

import paper_2511_09261_b200 as gnnco


_real_require = gnnco._require


class _Library:
    """Answers every call with OK (sizes with 4,096 bytes) and keeps the arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            if name.endswith("_bytes"):
                args[-1]._obj.value = 4096
            return 0
        return call

    def last(self, name):
        return [args for n, args in self.calls if n == name][-1]


@pytest.fixture
def graph(monkeypatch):
    g = gnnco.PartitionedGraph.__new__(gnnco.PartitionedGraph)
    g._lib, g._handle, g.device = _Library(), None, torch.device("cpu")
    g._plan_sizes, g._norm_sizes = {}, {}
    monkeypatch.setattr(gnnco, "_stream_ptr", lambda stream=None: 0 if stream is None else stream.cuda_stream)
    return g


def test_norm_gradients_have_a_work_area_per_call(graph, monkeypatch):
    """Calls on one stream, from two threads or while a graph is recorded, must not share partial sums."""
    kept, make = [], gnnco._empty
    monkeypatch.setattr(gnnco, "_empty", lambda *a: kept.append(make(*a)) or kept[-1])
    monkeypatch.setattr(gnnco, "_require", lambda t, *a: t)
    x, w = torch.ones(4, 8), torch.ones(8)
    areas = []
    for _ in range(2):
        graph.block_norm_backward(x, x.clone(), w)
        areas.append(graph._lib.last("gnnco_block_norm_backward")[3])
    assert areas[0] != areas[1]


class _Stream:
    def __init__(self, pointer):
        self.cuda_stream = pointer


class _Area:
    """Stands for a plan's work area; keeps the streams that it is said to be in use on."""
    device = torch.device("cpu")
    shape = (4096,)

    def __init__(self):
        self.used_on = []

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, stream):
        self.used_on.append(stream.cuda_stream)


def test_a_plan_used_on_another_stream_is_not_handed_out_again_before_that_use(graph, monkeypatch):
    monkeypatch.setattr(gnnco, "_require", lambda t, *a: t)
    monkeypatch.setattr(gnnco, "_empty", lambda *a: _Area())
    dout, out = torch.ones(6, 8), torch.empty(5, 8)
    tokens = torch.zeros(6, dtype=torch.int32)
    plan = graph.embedding_plan(tokens, 5, 8, stream=_Stream(17))
    graph.embedding_grad(plan, dout, out=out, stream=_Stream(17))
    assert plan.ws.used_on == []
    graph.embedding_grad(plan, dout, out=out, stream=_Stream(18))
    assert plan.ws.used_on == [18]
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream(0))
    graph.embedding_grad(plan, dout, out=out)
    assert plan.ws.used_on == [18, 0]


def test_work_areas_of_the_caller_are_checked(graph, monkeypatch):
    """An address that is not the handle's device's, or a count that is not bytes, must not reach the kernels."""
    monkeypatch.setattr(gnnco, "_require", lambda t, dtype, what, device="cuda": _real_require(t, dtype, what, "cpu"))
    G = torch.ones(2, 20, 24)
    area = torch.empty(8192, dtype=torch.uint8)
    for bad, error in ((torch.empty(8192), TypeError), (area[::2], TypeError), (1 << 20, TypeError),
                       (torch.empty(8192, dtype=torch.uint8, device="meta"), (TypeError, ValueError))):
        with pytest.raises(error):
            graph.orthogonalise(G, ws=bad)
        with pytest.raises(error):
            graph.muon_update(G.clone(), G.clone(), G, ws=bad)
    assert not [n for n, _ in graph._lib.calls if n in ("gnnco_orthogonalise", "gnnco_muon_update")]
    graph.orthogonalise(G, ws=area)
    assert graph._lib.last("gnnco_orthogonalise")[-3] == area.data_ptr()


def test_a_plan_of_another_device_is_refused(graph):
    plan = gnnco.EmbeddingPlan(6, 5, 8, torch.empty(4096, dtype=torch.uint8, device="meta"), 0)
    with pytest.raises(ValueError):
        graph.embedding_grad(plan, torch.ones(6, 8), out=torch.empty(5, 8))
    assert not graph._lib.calls


def test_a_step_of_another_number_of_layers_is_refused(graph, monkeypatch):
    """Gradients or momenta that do not go with the model's layers must not leave layers out silently."""
    from types import SimpleNamespace
    monkeypatch.setattr(gnnco, "_require", lambda t, *a: t)
    W = [torch.ones(2, 8, 4), torch.ones(2, 4, 1)]
    opt = SimpleNamespace(lr=0.1, momentum=0.9, nesterov=True, weight_decay=0.0, steps=5, coefs=gnnco.MUON_COEFS, eps=1e-7, active=None,
                          m=[torch.zeros_like(w) for w in W])
    model = SimpleNamespace(W=W)
    short = SimpleNamespace(**{**vars(opt), "m": opt.m[:1]})
    for o, dW in ((opt, W[:1]), (opt, W + W[:1]), (short, W)):
        with pytest.raises(ValueError):
            graph.muon_step(model, o, dW)
    assert not graph._lib.calls
    graph.muon_step(model, opt, W)
    assert sum(n == "gnnco_muon_update" for n, _ in graph._lib.calls) == 2


def test_sizes_past_32_bits_are_refused(graph, monkeypatch):
    """The C ABI counts table rows, columns and steps in 32 bits; what does not fit must not arrive as what is left of it."""
    monkeypatch.setattr(gnnco, "_require", lambda t, *a: t)
    graph.device = torch.device("meta")
    big = 2 ** 32 + 5
    tokens = torch.empty(6, dtype=torch.int32, device="meta")
    table = torch.empty(big, 8, dtype=torch.bfloat16, device="meta")
    wide = torch.empty(2, big, device="meta")
    tall = torch.empty(1, big, 3, device="meta")
    some = torch.empty(1, 4, 3, device="meta")
    for call in (lambda: graph.embedding_lookup(table, tokens), lambda: graph.embedding_lookup(wide, tokens),
                 lambda: graph.embedding_plan(tokens, big, 8), lambda: graph.embedding_plan(tokens, 8, big),
                 lambda: graph.block_norm(wide), lambda: graph.block_norm_backward(wide, wide),
                 lambda: graph.muon_update(tall, tall, tall), lambda: graph.orthogonalise(tall),
                 lambda: graph.orthogonalise(some, steps=big), lambda: graph.muon_update(some, some, some, steps=big)):
        with pytest.raises(ValueError):
            call()
    assert not graph._lib.calls


def test_results_without_their_inputs_are_refused(graph, monkeypatch):
    """A dy without y, or a dgate without a gate, would come back as it was given."""
    monkeypatch.setattr(gnnco, "_require", lambda t, *a: t)
    x = torch.ones(4, 8)
    for kw in (dict(dy=torch.empty(4, 8)), dict(dgate=torch.empty(8)), dict(y=x, dgate=torch.empty(4, 8))):
        with pytest.raises(ValueError):
            graph.block_norm_backward(x, x.clone(), **kw)
    assert not graph._lib.calls
