"""The operators around a training step, run together as examples/shared_embeddings.py does."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_lowers_the_loss_and_repeats_bit_for_bit(dtype):
    import torch
    import shared_embeddings as ex
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    totals, emb, grads = ex.train(30, feat_dtype=dt)
    assert totals[-1] < totals[0] and np.all(np.isfinite(totals))
    again, emb2, grads2 = ex.train(30, feat_dtype=dt)
    assert totals == again and torch.equal(emb.table, emb2.table)
    assert all(torch.equal(grads[k], grads2[k]) for k in grads)


def test_table_gradient_against_differences_of_the_loss():
    """Directional derivative of the loss through lookup, norms and the whole training step.  The loss is smooth in the
    table except where a hidden unit crosses zero; with steps of 1e-2 and less and gradients that float32 resolves to 1e-5, 3 %
    of the derivative (and 0.02 absolute, the float32 loss's own resolution over the step) covers both.  A step of 1e-2 along
    normals is 8 % of a table row, over which the norm bends: the central differences of two steps are extrapolated, which takes
    their leading error (the square of the step) out."""
    import torch
    import shared_embeddings as ex
    import paper_2511_09261_b200 as gnnco
    _, emb, _ = ex.train(1)
    graph, dev = emb.graph, emb.x.device
    import synth_inputs as si
    w = si.make_workload(1)
    W = [torch.from_numpy(w.weights(l)).to(dev) for l in range(w.L)]
    model = gnnco.Model(w.dims, W)
    dh = torch.empty_like(emb.x)
    graph.train_step(model, emb.forward(), ex.ALPHA, ex.BETA, dX=dh, flags=gnnco.WANT_DX)
    d = emb.backward(dh)["table"]
    v = torch.randn(d.shape, device=dev, generator=torch.Generator(device=dev).manual_seed(5))
    want = float((d.double() * v.double()).sum())
    start = emb.table.clone()

    def central(step):
        values = []
        for s in (step, -step):
            emb.table = start + s * v
            loss, _ = graph.train_step(model, emb.forward(), ex.ALPHA, ex.BETA, flags=gnnco.FORWARD_ONLY)
            values.append(float(loss.double().sum()))
        return (values[0] - values[1]) / (2 * step)

    slope = (4 * central(0.5e-2) - central(1e-2)) / 3
    assert abs(slope - want) <= 0.03 * abs(want) + 0.02, (slope, want)


def test_operators_are_counted_and_profiled():
    import torch
    import shared_embeddings as ex
    _, emb, _ = ex.train(1)
    graph = emb.graph
    before = graph.launch_count()
    graph.profile_begin()
    h = emb.forward()
    emb.backward(torch.ones_like(h))
    graph.muon_update(emb.table[None], emb.momentum[None], torch.ones_like(emb.table)[None])
    spent = graph.profile_end()
    assert graph.launch_count() > before
    assert {"embeddings", "block_norm", "muon"} <= set(spent) and all(ms > 0 for _, ms in spent.values())
