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
