"""Norms, gated feed-forward block, dropout and training step together, as examples/residual_block.py runs them."""
import os
import sys

import numpy as np
import pytest

import ff_ref
import paper_2511_09261_b200 as gnnco

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("p", [0.0, 0.1])
def test_the_example_runs(dtype, p):
    import torch
    import residual_block
    totals, block, grads = residual_block.train(4, p=p, feat_dtype=getattr(torch, dtype))
    assert np.all(np.isfinite(totals))
    assert all(bool(torch.isfinite(t).all()) for t in grads.values())
    assert all(bool(torch.isfinite(getattr(block, n)).all()) for n in ("w_gate", "w_up", "w_down", "gate"))


def _norm(v, w):
    import torch
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w


def test_gradients_of_the_whole_block():
    """float32: every gradient of the chain norm - block - norm against autograd in float64 on the CPU."""
    import torch
    import residual_block
    _, block, _ = residual_block.train(2, p=0.2)                  # weights and masks as training leaves them
    graph, n, F = block.graph, block.graph.n, block.x.shape[1]
    d_out = torch.randn(n, F, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    block.forward(block.x)
    got = block.backward(d_out)
    names = ("w_in", "w_post", "w_out", "gate", "w_gate", "w_up", "w_down")
    leaf = {k: getattr(block, k).double().cpu().requires_grad_(True) for k in names}
    leaf["x"] = block.x.double().cpu().requires_grad_(True)
    ptr = graph.arrays()["part_ptr"].cpu().tolist()
    h = _norm(leaf["x"], leaf["w_in"])
    parts = [(torch.nn.functional.silu(h[a:b] @ leaf["w_gate"][s]) * (h[a:b] @ leaf["w_up"][s])) @ leaf["w_down"][s]
             for s, (a, b) in enumerate(zip(ptr, ptr[1:]))]
    mask = ff_ref.keep(n, F, 0.2, 7, step=block.drop.step) / 0.8
    y = torch.cat(parts) * torch.from_numpy(mask)
    out = _norm(leaf["x"] + residual_block.RESIDUAL * leaf["gate"] * _norm(y, leaf["w_post"]), leaf["w_out"])
    out.backward(d_out.double().cpu())
    for k, v in leaf.items():
        # float32 chains of sums over at most 125 rows or 96 columns: some 200 roundings of 2^-24, by norm
        err = (got[k].double().cpu() - v.grad).norm() / v.grad.norm()
        assert float(err) < 200 * 2.0 ** -24, (k, float(err))


def test_a_step_with_the_block_recorded_and_replayed():
    """Forward and backward of the block in one graph whose masks advance with a device counter, against eager calls."""
    import torch
    import residual_block
    _, block, _ = residual_block.train(1, p=0.1)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    block.drop = gnnco.Dropout(0.3, 99, layer=1, step_dev=step)
    x, d_out = block.x, torch.randn_like(block.x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        block.forward(x)
        block.backward(d_out)
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        out = block.forward(x)
        grads = block.backward(d_out)
        step.add_(1)
    eager = residual_block.ResidualBlock(block.graph, x.shape[1], 96)
    for name in ("w_gate", "w_up", "w_down", "w_in", "w_post", "w_out", "gate"):
        setattr(eager, name, getattr(block, name))
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        eager.drop = gnnco.Dropout(0.3, 99, layer=1, step=k)
        want = eager.forward(x)
        assert torch.equal(out, want)
        want_grads = eager.backward(d_out)
        assert all(torch.equal(grads[n], want_grads[n]) for n in grads)


def test_two_threads_and_streams_at_once():
    """Blocks of two models on one handle, issued by two threads on streams of their own."""
    import threading
    import torch
    import residual_block
    _, block, _ = residual_block.train(1)
    graph, x = block.graph, block.x
    other = residual_block.ResidualBlock(graph, x.shape[1], 200, act="gelu", seed=8)
    d_out = torch.randn_like(x)

    def run(b):
        return [b.forward(x), *b.backward(d_out).values()]
    want = [run(block), run(other)]
    torch.cuda.synchronize()
    got = [None, None]

    def work(i, b):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got[i] = run(b)
        s.synchronize()
    threads = [threading.Thread(target=work, args=(i, b)) for i, b in enumerate((block, other))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
