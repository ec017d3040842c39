"""Orthogonalised updates of more matrices than the GPU works on at once: every CTA (pair, warp) takes several, with
gaps in `active` between them."""
import numpy as np
import pytest

import operators_ref as ref
from helpers import tiny_graph
from gpu_common import load_graph

pytestmark = pytest.mark.gpu
COEFS = (3.4445, -4.7750, 2.0315)
# rounding errors of 2^-24 grow by a = 3.4445 per step in the worst direction: 2^-24 * 3.4445^5 * sqrt(15 products)
O_RTOL = 1.1e-4


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _normal(seed, *shape):
    import torch
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _by_few(graph, G, few, **kw):
    """The same matrices in calls of `few` sets: no CTA takes a second matrix."""
    import torch
    return torch.cat([graph.orthogonalise(G[s:s + few].contiguous(), **kw) for s in range(0, G.shape[0], few)])


def _near(got, G, sample, eps):
    """Some sets against the definition in float64."""
    for s in sample:
        want = ref.newton_schulz(G[s:s + 1].cpu().numpy(), 5, COEFS, eps)[0]
        err = np.sqrt(((got[s].double().cpu().numpy() - want) ** 2).sum())
        assert err <= O_RTOL * np.sqrt((want ** 2).sum()), (s, err)


@pytest.mark.parametrize("sets,r,c", [(230, 130, 140), (310, 40, 200), (620, 100, 48)])
def test_norms_that_are_summed_twice(graph, sets, r, c):
    """Matrices whose squares leave float32's range take their norm in a second round; here all, some and none of those that
    follow one another in a CTA or pair."""
    import torch
    G = _normal(1, sets, r, c)
    exponents = torch.tensor([2.0 ** -60, 1.0, 2.0 ** 80, 2.0 ** 80, 1.0], device="cuda")
    G *= exponents[torch.arange(sets, device="cuda") * 7 // 5 % 5][:, None, None]
    eps = 1e-30
    got = graph.orthogonalise(G, coefs=COEFS, eps=eps)
    assert torch.equal(got, _by_few(graph, G, 50, coefs=COEFS, eps=eps))
    _near(got, G, (0, 1, 2, 3, sets // 2, sets - 1), eps)
    assert graph.async_status() == 0


@pytest.mark.parametrize("sets,r,c", [(700, 17, 20), (700, 32, 32), (650, 64, 24), (650, 32, 100), (400, 24, 180), (330, 150, 20)])
def test_matrices_that_leave_warps_idle(graph, sets, r, c):
    """Sides that fill neither the 128 rows nor the 32-column items of all working warps."""
    import torch
    G = _normal(2, sets, r, c)
    got = graph.orthogonalise(G, coefs=COEFS, eps=1e-7)
    assert torch.equal(got, _by_few(graph, G, 130, coefs=COEFS, eps=1e-7))
    _near(got, G, (0, 1, sets // 2, sets - 1), 1e-7)
    assert graph.async_status() == 0
