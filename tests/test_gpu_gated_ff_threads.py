"""The block on a handle whose training step another thread is issuing: the step's exchange of tables must not reach it."""
import threading

import numpy as np
import pytest

import paper_2511_09261_b200 as gnnco
from gpu_common import load_graph, to_dev
from helpers import rand_features, rand_weights, tiny_graph

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_block_beside_steps_on_some_subgraphs(dtype):
    import torch
    dt = getattr(torch, dtype)
    eu, ev, part = tiny_graph(3000, 0.003, 6, seed=31)
    S = int(part.max()) + 1
    graph = load_graph(3000, eu, ev, part, S)
    dims = [64, 32, 1]
    X = to_dev(rand_features(3000, 64, 3).astype(np.float32)).to(dt)
    W = [to_dev(w.astype(np.float32)) for w in rand_weights(dims, S, 7)]
    model = gnnco.Model(dims, W, gnnco.BF16 if dt == torch.bfloat16 else gnnco.F32)
    opt = gnnco.Adam(model, lr=0.0)                              # (the weights stay, so every step has the same results)
    opt.active = to_dev(np.array([0, 1, 0, 0, 1, 0], np.uint8))
    graph.active_plan(opt.active)
    r = torch.Generator(device="cuda").manual_seed(2)
    w = [torch.randn(s, device="cuda", generator=r).mul_(0.1).to(dt) for s in ((S, 64, 96), (S, 64, 96), (S, 96, 64))]
    dy = torch.randn(3000, 64, device="cuda", generator=r).to(dt)

    def block():
        return [graph.gated_ff(X, *w), *graph.gated_ff_backward(X, dy, *w).values()]

    def step():
        return graph.train_step(model, X, 2.0, 1.0, opt=opt, flags=gnnco.ACTIVE_ONLY)[1]
    want, want_p = block(), step()
    torch.cuda.synchronize()
    got, last, done, errors = [], [want_p], threading.Event(), []

    def train():
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(4000):
                    if done.is_set():
                        break
                    last[0] = step()
            s.synchronize()
        except Exception as e:                                    # told to the thread that asserts
            errors.append(e)
    t = threading.Thread(target=train)
    t.start()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(200):
            got.append(block())
    s.synchronize()
    done.set()
    t.join()
    assert not errors, errors
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    active = torch.from_numpy(np.isin(np.sort(part), [1, 4])).cuda()
    assert torch.equal(last[0][active], want_p[active])
    assert graph.async_status() == gnnco.OK
