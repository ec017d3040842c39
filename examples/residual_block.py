"""Training with a residual block in front of the GCN: norms, a gated feed-forward block per subgraph, dropout.

A step runs

    norm            h  = norm(x) w_in                                    gnnco_block_norm
    block           y  = drop((act(h Wg) .* (h Wu)) Wd), a set of weights per subgraph      gnnco_gated_ff
    norm            x' = x + g .* norm(y) w_post,  h' = norm(x') w_out   gnnco_block_norm
    training step   loss, dW, dh' from h' (WANT_DX)                      gnnco_train_step
    backward        dy, dx', .. from dh'; dh, dWg, dWu, dWd from dy; dx  gnnco_block_norm_backward, gnnco_gated_ff_backward
    updates         orthogonalised for the matrices, plain for the vectors   gnnco_muon_update

with x the fixed random embeddings of the nodes (its gradient is there for what may come before).  Nothing but h, y and x' is kept
for the backward pass: g, u and the dropout mask are computed again.  Run it with  python examples/residual_block.py [steps].
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2511_09261_b200 as gnnco
import synth_inputs as si

ALPHA, BETA, RESIDUAL = 2.0, 1.0, 0.5


class ResidualBlock:
    """The block's weights (float32 masters, also for bfloat16 features) and what its backward pass needs."""

    def __init__(self, graph, F, H, act="silu", p=0.1, seed=7):
        g = torch.Generator(device=graph.device).manual_seed(1)
        draw = lambda scale, *shape: torch.randn(*shape, device=graph.device, generator=g) * scale  # noqa: E731
        self.graph, self.act = graph, act
        self.w_gate, self.w_up = draw(F ** -0.5, graph.S, F, H), draw(F ** -0.5, graph.S, F, H)
        self.w_down = draw(H ** -0.5, graph.S, H, F)
        self.momenta = [torch.zeros_like(w) for w in (self.w_gate, self.w_up, self.w_down)]
        self.w_in, self.w_post, self.w_out = (torch.ones(F, device=graph.device) for _ in range(3))
        self.gate = torch.full((F,), 0.5, device=graph.device)
        self.drop = gnnco.Dropout(p, seed) if p else None

    def forward(self, x):
        self.x = x
        _, self.h = self.graph.block_norm(x, self.w_in)
        self.y = self.graph.gated_ff(self.h, self.w_gate, self.w_up, self.w_down, act=self.act, drop=self.drop)
        self.stream, out = self.graph.block_norm(x, self.w_out, y=self.y, w_post=self.w_post, gate=self.gate, scale=RESIDUAL)
        return out

    def backward(self, d_out):
        d = self.graph.block_norm_backward(self.stream, d_out, self.w_out, y=self.y, w_post=self.w_post, gate=self.gate,
                                           scale=RESIDUAL)
        f = self.graph.gated_ff_backward(self.h, d["dy"], self.w_gate, self.w_up, self.w_down, act=self.act, drop=self.drop)
        e = self.graph.block_norm_backward(self.x, f["dx"], self.w_in, dx_out=d["dx"])
        return dict(x=e["dx"], w_in=e["dw_pre"], w_out=d["dw_pre"], w_post=d["dw_post"], gate=d["dgate"], w_gate=f["dw_gate"],
                    w_up=f["dw_up"], w_down=f["dw_down"])

    def update(self, d, lr):
        for name, m in zip(("w_gate", "w_up", "w_down"), self.momenta):
            self.graph.muon_update(getattr(self, name), m, d[name], lr=lr)
        for name in ("w_in", "w_post", "w_out", "gate"):
            getattr(self, name).sub_(d[name], alpha=lr / self.graph.n)
        if self.drop:
            self.drop.step += 1                                   # a new mask for the next step


def train(steps=40, lr=0.02, hidden=96, p=0.1, feat_dtype=None):
    """Total loss per step on the 1,000-node Erdos-Renyi graph (8 subgraphs, widths 64-32-1)."""
    feat_dtype = feat_dtype or torch.float32
    w = si.make_workload(1)
    dev = torch.device("cuda", torch.cuda.current_device())
    graph = gnnco.gnnco_partition_load(*(torch.from_numpy(a).to(dev) for a in (w.eu, w.ev, w.part)), w.S)
    x = torch.from_numpy(w.features_f32()).to(dev)[graph.arrays()["perm"].long()].to(feat_dtype)
    block = ResidualBlock(graph, x.shape[1], hidden, p=p)
    W = [torch.from_numpy(w.weights(l)).to(dev) for l in range(w.L)]
    model = gnnco.Model(w.dims, W, gnnco.BF16 if feat_dtype == torch.bfloat16 else gnnco.F32)
    opt = gnnco.Muon(model, lr=lr)
    dW, dh = [torch.empty_like(v) for v in W], torch.empty_like(x)
    losses = []
    for _ in range(steps):
        loss, _p = graph.train_step(model, block.forward(x), ALPHA, BETA, dW=dW, dX=dh, flags=gnnco.WANT_DX)
        grads = block.backward(dh)
        graph.muon_step(model, opt, dW)
        block.update(grads, lr)
        losses.append(loss.sum())
    assert graph.async_status() == gnnco.OK
    return torch.stack(losses).tolist(), block, grads


if __name__ == "__main__":
    totals, _, _ = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    print("total loss %.3f -> %.3f" % (totals[0], totals[-1]))
