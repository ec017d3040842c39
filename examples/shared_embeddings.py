"""Training with input embeddings that nodes share.

Every node of a graph carries a token -- here its degree class -- and learns through one row of a small table instead of
a row of its own.  A step runs

    lookup          y  = s * table[token]                         gnnco_embedding_lookup
    norms           x' = x + g .* norm(y) w_post, h = norm(x') w_pre   gnnco_block_norm
    training step   loss, dW, dh from h (WANT_DX)                 gnnco_train_step
    backward        dy, dg, dw_post, dw_pre from dh               gnnco_block_norm_backward
    table gradient  dtable from dy, rows in token order           gnnco_embedding_grad
    updates         orthogonalised for weights and table, plain for the vectors   gnnco_muon_update

with x the fixed random embeddings of the nodes.  Run it with  python examples/shared_embeddings.py [steps].
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2511_09261_b200 as gnnco
import synth_inputs as si

ALPHA, BETA, RESIDUAL = 2.0, 1.0, 0.5


class SharedEmbeddings:
    """The table, the two norms and the gate, and what their backward pass needs."""

    def __init__(self, graph, tokens, V, x):
        self.graph, self.tokens, self.V, self.x = graph, tokens, V, x
        F = x.shape[1]
        self.plan = graph.embedding_plan(tokens, V, F)            # the tokens do not change: ordered once
        g = torch.Generator(device=x.device).manual_seed(1)
        self.table = torch.randn(V, F, device=x.device, generator=g) * F ** -0.5
        self.momentum = torch.zeros_like(self.table)
        self.scale = F ** 0.5
        self.w_pre, self.w_post = torch.ones(F, device=x.device), torch.ones(F, device=x.device)
        self.gate = torch.full((F,), 0.5, device=x.device)

    def forward(self):
        self.y = self.graph.embedding_lookup(self.table, self.tokens, scale=self.scale, out_dtype=self.x.dtype)
        self.stream, h = self.graph.block_norm(self.x, self.w_pre, y=self.y, w_post=self.w_post, gate=self.gate, scale=RESIDUAL)
        return h

    def backward(self, dh):
        d = self.graph.block_norm_backward(self.stream, dh, self.w_pre, y=self.y, w_post=self.w_post, gate=self.gate,
                                           scale=RESIDUAL)
        d["table"] = self.graph.embedding_grad(self.plan, d["dy"], scale=self.scale)
        return d

    def update(self, d, lr):
        n = self.x.shape[0]
        self.graph.muon_update(self.table[None], self.momentum[None], d["table"][None], lr=lr)
        for p, name in ((self.w_pre, "dw_pre"), (self.w_post, "dw_post"), (self.gate, "dgate")):
            p.sub_(d[name], alpha=lr / n)


def train(steps=40, seed=3, lr=0.02, feat_dtype=None):
    """Total loss per step on the 1,000-node Erdos-Renyi graph (8 subgraphs, widths 64-32-1)."""
    feat_dtype = feat_dtype or torch.float32
    w = si.make_workload(1)
    dev = torch.device("cuda", torch.cuda.current_device())
    graph = gnnco.gnnco_partition_load(*(torch.from_numpy(a).to(dev) for a in (w.eu, w.ev, w.part)), w.S)
    view = graph.arrays()
    degree = view["rowptr"][1:] - view["rowptr"][:-1]             # new node order, like X
    V = int(degree.max()) + 1
    x = torch.from_numpy(w.features_f32()).to(dev)[view["perm"].long()].to(feat_dtype)
    emb = SharedEmbeddings(graph, degree.to(torch.int32).contiguous(), V, x)
    W = [torch.from_numpy(w.weights(l)).to(dev) for l in range(w.L)]
    model = gnnco.Model(w.dims, W, gnnco.BF16 if feat_dtype == torch.bfloat16 else gnnco.F32)
    opt = gnnco.Muon(model, lr=lr)
    dW, dh = [torch.empty_like(v) for v in W], torch.empty_like(x)
    losses = []
    for _ in range(steps):
        loss, _p = graph.train_step(model, emb.forward(), ALPHA, BETA, dW=dW, dX=dh, flags=gnnco.WANT_DX)
        grads = emb.backward(dh)
        graph.muon_step(model, opt, dW)
        emb.update(grads, lr)
        losses.append(loss.sum())
    assert graph.async_status() == gnnco.OK
    return torch.stack(losses).tolist(), emb, grads


if __name__ == "__main__":
    totals, emb, _ = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    print("%d tokens; total loss %.3f -> %.3f" % (emb.V, totals[0], totals[-1]))
