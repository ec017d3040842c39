"""Orthogonalised updates on the GPU against the float64 restatement."""
import numpy as np
import pytest

import operators_ref as ref
from helpers import tiny_graph
from gpu_common import load_graph, to_dev

pytestmark = pytest.mark.gpu
COEFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
# Error of the iterate.  A rounding error of 2^-24 (relative to |X|_F = 1, what the iteration starts from) in the direction
# of a small singular value grows by a = 3.4445 per step, 3.4445^5 = 485 in all; the 15 products of five steps add errors of
# that size, 2^-24 * 485 * sqrt(15) = 1.1e-4 of |O|_F if every one of them met the worst direction.
O_RTOL = 1.1e-4
SIZES = [(1, 1, 1), (2, 1, 7), (2, 9, 1), (3, 8, 8), (2, 16, 33), (1, 33, 16), (5, 64, 32), (2, 32, 64), (2, 65, 63), (3, 100, 128),
         (2, 128, 128), (3, 129, 128), (2, 128, 130), (1, 120, 256), (2, 256, 100), (1, 128, 257), (1, 300, 128), (2, 130, 200),
         (2, 200, 200), (3, 256, 256), (1, 257, 255), (1, 257, 300), (1, 384, 320), (1, 513, 640)]


@pytest.fixture(scope="module")
def graph():
    eu, ev, part = tiny_graph(64, 0.1, 2, seed=5)
    return load_graph(64, eu, ev, part, int(part.max()) + 1)


def _grad(seed, sets, r, c, scale=1e-2):
    """A few strong directions over noise."""
    rng = np.random.RandomState(seed)
    k = min(4, r, c)
    g = rng.standard_normal((sets, r, k)) @ rng.standard_normal((sets, k, c)) + 0.5 * rng.standard_normal((sets, r, c))
    return (scale * g).astype(np.float32)


def _near(got, want, extra=0.0):
    err = np.sqrt(((got - want) ** 2).sum(axis=(1, 2)))
    size = np.sqrt((want ** 2).sum(axis=(1, 2)))
    assert np.all(err <= (O_RTOL + extra) * size + 1e-30), (err / size).max()


@pytest.mark.parametrize("sets,r,c", SIZES)
@pytest.mark.parametrize("gd,od", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_orthogonalise(graph, sets, r, c, gd, od):
    import torch
    dt = dict(f32=torch.float32, bf16=torch.bfloat16)
    G = torch.from_numpy(_grad(1, sets, r, c)).to(dt[gd])
    got = graph.orthogonalise(G.cuda(), out_dtype=dt[od], coefs=COEFS, eps=EPS)
    assert got.dtype == dt[od]
    want = ref.newton_schulz(G.float().numpy(), 5, COEFS, EPS)
    _near(got.double().cpu().numpy(), want, 2.0 ** -8 if od == "bf16" else 0.0)


@pytest.mark.parametrize("sets,r,c", SIZES)
@pytest.mark.parametrize("nesterov", [True, False])
def test_update(graph, sets, r, c, nesterov):
    import torch
    rng = np.random.RandomState(2)
    W, m, g = rng.standard_normal((sets, r, c)).astype(np.float32), _grad(3, sets, r, c), _grad(4, sets, r, c)
    f32 = lambda v: float(np.float32(v))  # noqa: E731  (the library receives float32 hyper-parameters)
    Wd, md = to_dev(W), to_dev(m)
    graph.muon_update(Wd, md, to_dev(g), lr=0.3, momentum=0.9, nesterov=nesterov, weight_decay=0.1, coefs=COEFS, eps=EPS)
    Wr, mr = ref.muon(W, m, g, f32(0.3), f32(0.9), nesterov, f32(0.1), 5, [f32(v) for v in COEFS], EPS)
    # m: a product and a sum in float32
    assert np.all(np.abs(md.cpu().numpy() - mr) <= 2.0 ** -23 * (np.abs(0.9 * m) + np.abs(g)))
    # W: the step inherits the iterate's error, and the product and the sum round (lr and decay are float32 products too)
    step = np.abs(Wr - W)
    err = np.sqrt(((Wd.double().cpu().numpy() - Wr) ** 2).sum(axis=(1, 2)))
    size = np.sqrt((step ** 2).sum(axis=(1, 2)))
    assert np.all(err <= 1.2 * O_RTOL * size + 2.0 ** -22 * np.sqrt((W ** 2).sum(axis=(1, 2)))), err / size


def test_inactive_sets_are_untouched_and_sets_do_not_depend_on_their_number(graph):
    import torch
    for r, c in ((24, 40), (128, 128), (200, 256), (300, 300)):
        sets = 7
        W, m, g = to_dev(_grad(1, sets, r, c)), to_dev(_grad(2, sets, r, c)), to_dev(_grad(3, sets, r, c))
        W1, m1 = W.clone(), m.clone()
        graph.muon_update(W1, m1, g, coefs=COEFS)
        W2, m2 = W.clone(), m.clone()
        active = to_dev(np.array([1, 0, 1, 1, 0, 0, 1], np.uint8))
        graph.muon_update(W2, m2, g, coefs=COEFS, active=active)
        on = active.bool()
        assert torch.equal(W2[on], W1[on]) and torch.equal(m2[on], m1[on])
        assert torch.equal(W2[~on], W[~on]) and torch.equal(m2[~on], m[~on])
        for s in (0, 6):
            W3, m3 = W[s:s + 1].clone(), m[s:s + 1].clone()
            graph.muon_update(W3, m3, g[s:s + 1].contiguous(), coefs=COEFS)
            assert torch.equal(W3[0], W1[s]) and torch.equal(m3[0], m1[s])
        O = torch.full_like(g, 5.0)
        graph.orthogonalise(g, out=O, active=active)
        assert bool((O[~on] == 5.0).all()) and torch.equal(O[on], graph.orthogonalise(g)[on])


@pytest.mark.parametrize("r,c", [(16, 16), (128, 100), (256, 256), (300, 260)])
def test_zero_tiny_huge_and_broken_gradients(graph, r, c):
    import torch
    G = torch.from_numpy(_grad(5, 6, r, c)).cuda()
    G[0] = 0.0
    G[1] *= 1e-12                                # |u| far below eps: the iterate stays small but is not zero
    G[2] *= 1e30                                 # squares past float32
    G[3, 0, 0] = float("inf")
    G[4, r - 1, c - 1] = float("nan")
    O = graph.orthogonalise(G, coefs=COEFS, eps=EPS).cpu().numpy()
    assert np.all(O[0] == 0)
    want = ref.newton_schulz(G.cpu().numpy()[[1, 2, 5]], 5, COEFS, EPS)
    _near(O[[1, 2, 5]].astype(np.float64), want)
    assert np.isnan(O[3]).any() and np.isnan(O[4]).any()


@pytest.mark.parametrize("steps,coefs", [(1, (1.5, -0.5, 0.0)), (12, (1.5, -0.5, 0.0)), (32, (2.0, -1.5, 0.5)), (3, (0.5, 0.25, -0.125))])
def test_other_coefficients(graph, steps, coefs):
    for r, c in ((40, 30), (256, 130), (260, 300)):
        G = _grad(6, 2, r, c)
        O = graph.orthogonalise(to_dev(G), steps=steps, coefs=coefs, eps=EPS).double().cpu().numpy()
        want = ref.newton_schulz(G, steps, coefs, EPS)
        # the same bound: growth per step is at most 2, and converged directions stop growing
        err = np.sqrt(((O - want) ** 2).sum(axis=(1, 2))) / np.sqrt((want ** 2).sum(axis=(1, 2)))
        assert np.all(err <= 2.0 ** -24 * min(2.0 ** steps, 4 * max(r, c)) * np.sqrt(3 * steps) + 2.0 ** -20), err


def test_in_place_workspace_and_streams(graph):
    import torch
    G = to_dev(_grad(7, 4, 256, 200))
    want = graph.orthogonalise(G)
    buf = G.clone()
    assert graph.orthogonalise(buf, out=buf) is buf and torch.equal(buf, want)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda").random_(0, 256)     # left-overs must not matter
    assert torch.equal(graph.orthogonalise(G, ws=ws), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    O = graph.orthogonalise(G, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(O, want)


def test_bf16_weight_copies_are_rebuilt_after_an_update():
    """A step that may reuse the bf16 copies of the weights must notice that an update has changed the weights."""
    import torch
    import paper_2511_09261_b200 as gnnco
    eu, ev, part = tiny_graph(300, 0.05, 2, seed=9)
    g = load_graph(300, eu, ev, part, 2)
    dims = [64, 64, 1]
    rng = np.random.RandomState(1)
    X = to_dev(rng.standard_normal((300, 64)).astype(np.float32)).bfloat16()
    losses = []
    for flag in (0, gnnco.WEIGHTS_UNTOUCHED):
        W = [to_dev((0.2 * rng.standard_normal((2, a, b))).astype(np.float32)) for a, b in zip(dims, dims[1:])]
        rng = np.random.RandomState(1)
        W = [to_dev((0.2 * rng.standard_normal((2, a, b))).astype(np.float32)) for a, b in zip(dims, dims[1:])]
        model = gnnco.Model(dims, W, gnnco.BF16)
        adam, muon = gnnco.Adam(model, lr=1e-2), gnnco.Muon(model, lr=0.1)
        dW = [torch.empty_like(w) for w in W]
        out = []
        for _ in range(3):
            loss, _p = g.train_step(model, X, 2.0, 1.0, opt=adam, dW=dW, flags=flag)
            out.append(loss.clone())
            g.muon_step(model, muon, dW)
        losses.append(torch.stack(out))
    assert torch.equal(losses[0], losses[1])


def test_refusals(graph):
    import torch
    import paper_2511_09261_b200 as gnnco
    G = torch.ones(2, 8, 4, device="cuda")
    for call in (lambda: graph.orthogonalise(G.half()), lambda: graph.orthogonalise(G.transpose(1, 2)), lambda: graph.orthogonalise(G.cpu()),
                 lambda: graph.muon_update(G.clone(), G.clone(), G.bfloat16())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: graph.orthogonalise(G[0]), lambda: graph.orthogonalise(G, out=torch.empty(2, 4, 8, device="cuda")),
                 lambda: graph.muon_update(G.clone(), G[:1].clone(), G),
                 lambda: graph.orthogonalise(G, active=torch.ones(3, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for bad in (dict(steps=0), dict(steps=33), dict(eps=0.0), dict(coefs=(9.0, 1.0, 1.0)), dict(coefs=(float("nan"), 0.0, 0.0))):
        with pytest.raises(gnnco.GnncoError) as e:
            graph.orthogonalise(G, **bad)
        assert e.value.status == gnnco.INVALID_ARGUMENT
    big = torch.ones(1, 300, 300, device="cuda")
    with pytest.raises(gnnco.GnncoError) as e:
        graph.orthogonalise(big, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == gnnco.WORKSPACE_TOO_SMALL
