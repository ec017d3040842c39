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


def _update_by_few(graph, W, m, g, few, active):
    import torch
    W, m = W.clone(), m.clone()
    for s in range(0, W.shape[0], few):
        part = slice(s, s + few)
        graph.muon_update(W[part], m[part], g[part], coefs=COEFS, weight_decay=0.1, active=active[part].contiguous())
    return W, m


@pytest.mark.parametrize("sets,r,c,few", [
    (700, 32, 32, 130), (650, 128, 100, 130), (400, 40, 200, 130), (310, 200, 70, 130),      # one CTA each, one or two per SM
    (200, 130, 140, 50), (180, 256, 256, 50), (160, 200, 131, 50),                           # pairs
    (20_000, 16, 9, 4000), (12_000, 1, 40, 4000), (10_000, 40, 16, 4000),                    # warps
    (120, 260, 300, 40), (300, 30, 270, 70),                                                 # tiles: chunks of 99 and of 592 sets
])
def test_many_sets_with_gaps(graph, sets, r, c, few):
    """Sets 0, 1, .. take turns in being left out in ways that no number of CTAs divides; one stretch of 100 is out altogether."""
    import torch
    W, m, g = _normal(1, sets, r, c), _normal(2, sets, r, c), _normal(3, sets, r, c)
    at = torch.arange(sets, device="cuda")
    on = ((at * 5) % 7 < 4) & ~((at >= sets // 3) & (at < sets // 3 + min(100, sets // 4)))
    active = on.to(torch.uint8)
    W1, m1 = W.clone(), m.clone()
    graph.muon_update(W1, m1, g, coefs=COEFS, weight_decay=0.1, active=active)
    W2, m2 = _update_by_few(graph, W, m, g, few, active)
    assert torch.equal(W1, W2) and torch.equal(m1, m2)
    assert torch.equal(W1[~on], W[~on]) and torch.equal(m1[~on], m[~on])
    f32 = lambda v: float(np.float32(v))  # noqa: E731
    picked = torch.nonzero(on)[:, 0]
    for s in [int(picked[i]) for i in (0, 1, len(picked) // 2, -2, -1)]:
        one = slice(s, s + 1)
        Wr, _ = ref.muon(*(t[one].cpu().numpy() for t in (W, m, g)), f32(0.02), f32(0.95), True, f32(0.1), 5, [f32(v) for v in COEFS], 1e-7)
        w = W[one].cpu().numpy()
        err, step = np.sqrt(((W1[one].double().cpu().numpy() - Wr) ** 2).sum()), np.sqrt(((Wr - w) ** 2).sum())
        # the iterate's error, and the roundings of a product, a sum and two float32 factors
        assert err <= 1.2 * O_RTOL * step + 2.0 ** -22 * np.sqrt((w.astype(np.float64) ** 2).sum()), (s, err)
    assert graph.async_status() == 0


@pytest.mark.parametrize("r,c,counts", [
    (64, 2700, (1, 60, 100)),            # a cluster per tile of X X^T, narrow tiles, wide tiles
    (2700, 100, (1, 100)),               # the same from the other side
    (300, 2600, (1, 10, 30)),            # six tiles of X X^T per matrix
    (300, 300, (1, 30)),                 # narrow and wide tiles
    (257, 700, (1, 40)),
])
def test_all_tile_forms_give_the_same_bits(graph, r, c, counts):
    import torch
    G = _normal(4, max(counts), r, c)
    want = graph.orthogonalise(G[:1].contiguous(), coefs=COEFS, eps=1e-7)
    _near(want, G, (0,), 1e-7)
    for n in counts[1:]:
        got = graph.orthogonalise(G[:n].contiguous(), coefs=COEFS, eps=1e-7)
        assert torch.equal(got[:1], want)
        last = graph.orthogonalise(G[n - 1:n].contiguous(), coefs=COEFS, eps=1e-7)
        assert torch.equal(got[n - 1:], last)
        _near(got, G, (n - 1,), 1e-7)
    assert graph.async_status() == 0
