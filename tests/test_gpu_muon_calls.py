"""Calls of the orthogonalised updates beside the ordinary ones: parts of a layer's weights, tiny eps, work areas."""
import numpy as np
import pytest

from helpers import tiny_graph
from gpu_common import load_graph, to_dev

pytestmark = pytest.mark.gpu
COEFS = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


@pytest.mark.parametrize("write", ["first sets", "last sets", "middle", "iterate"])
def test_bf16_copies_are_rebuilt_after_a_part_of_the_weights_changed(write):
    """A step that may reuse the bf16 copies of the weights notices that some sets of a layer have changed."""
    import torch
    import paper_2511_09261_b200 as gnnco
    eu, ev, part = tiny_graph(300, 0.05, 5, seed=9)
    g = load_graph(300, eu, ev, part, 5)
    dims = [64, 64, 1]
    X = to_dev(np.random.RandomState(1).standard_normal((300, 64)).astype(np.float32)).bfloat16()
    lo, hi = {"first sets": (0, 2), "last sets": (3, 5), "middle": (1, 4), "iterate": (1, 2)}[write]
    losses = []
    for flag in (0, gnnco.WEIGHTS_UNTOUCHED):
        rng = np.random.RandomState(2)
        W = [to_dev((0.2 * rng.standard_normal((5, a, b))).astype(np.float32)) for a, b in zip(dims, dims[1:])]
        model = gnnco.Model(dims, W, gnnco.BF16)
        adam = gnnco.Adam(model, lr=1e-2)
        dW = [torch.empty_like(w) for w in W]
        out = []
        for _ in range(3):
            loss, _p = g.train_step(model, X, 2.0, 1.0, opt=adam, dW=dW, flags=flag)
            out.append(loss.clone())
            some = W[0][lo:hi]
            if write == "iterate":
                g.orthogonalise(dW[0][lo:hi], out=some)
            else:
                g.muon_update(some, torch.zeros_like(some), dW[0][lo:hi], lr=0.1)
        losses.append(torch.stack(out))
    assert not torch.equal(losses[0][0], losses[0][1])
    assert torch.equal(losses[0], losses[1])


@pytest.mark.parametrize("r,c", [(16, 16), (1, 9), (128, 100), (100, 200), (200, 256), (300, 260)])
@pytest.mark.parametrize("eps", [1e-36, 1e-42])
def test_any_eps_above_zero(graph, r, c, eps):
    """A zero gradient stays zero, and one far below float32's normal range is orthogonalised like any other.  (2^-24 grows by 3.4445
    per step: 1.1e-4 over the 15 products of five steps in the worst direction; entries below 2^-126 are given as they are.)"""
    import torch
    import operators_ref as ref
    G = torch.randn(3, r, c, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    G[0] = 0.0
    G[1] *= 1e-37
    O = graph.orthogonalise(G, coefs=COEFS, eps=eps)
    assert bool((O[0] == 0).all())
    want = ref.newton_schulz(G[1:].cpu().numpy(), 5, COEFS, float(np.float32(eps)))
    err = np.sqrt(((O[1:].double().cpu().numpy() - want) ** 2).sum(axis=(1, 2)))
    assert np.all(err <= 1.1e-4 * np.sqrt((want ** 2).sum(axis=(1, 2)))), err
    W, m = torch.ones(3, r, c, device="cuda"), torch.zeros(3, r, c, device="cuda")
    graph.muon_update(W, m, torch.zeros_like(W), eps=eps)
    assert bool((W == 1).all()) and bool((m == 0).all())


def test_no_work_area_where_none_is_needed(graph):
    import torch
    import paper_2511_09261_b200 as gnnco
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    for r, c in ((16, 9), (128, 100), (90, 250)):
        G = torch.randn(3, r, c, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        assert torch.equal(graph.orthogonalise(G, ws=none), graph.orthogonalise(G))
        W, W2 = torch.ones_like(G), torch.ones_like(G)
        graph.muon_update(W, torch.zeros_like(G), G, ws=none)
        graph.muon_update(W2, torch.zeros_like(G), G)
        assert torch.equal(W, W2)
    for r, c in ((200, 200), (300, 300)):
        with pytest.raises(gnnco.GnncoError) as e:
            graph.orthogonalise(torch.ones(1, r, c, device="cuda"), ws=none)
        assert e.value.status == gnnco.WORKSPACE_TOO_SMALL
