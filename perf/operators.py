"""Timed cases of the operators around a training step: shared input embeddings (lookup and gradient), the norms
before and after a residual block, and weight updates orthogonalised by Newton-Schulz products.

With ``own = False`` a case runs in its plain form, elementary torch operations in float32; with ``own = True`` it runs
through the entry points of ``paper_2511_09261_b200``.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFS = (3.4445, -4.7750, 2.0315)          # odd quintic of the Newton-Schulz iteration
NS_STEPS, NS_EPS = 5, 1e-7
NORM_EPS = 1e-6


def listed():
    return [
        # the 1,000-node graph: every node carries one of 32 structure classes; a call of a few microseconds
        dict(name="lookup-1k", op="lookup", rows=1000, V=32, F=64, dtype="f32"),
        # the 10,000,000-node graph in bfloat16, width 256: the table lives in L2, the output is 5 GB
        dict(name="lookup-10m", op="lookup", rows=10_000_000, V=100_000, F=256, dtype="bf16"),
        # gradient of the table on the social-ego-network shape: 4,039 nodes, odd vocabulary
        dict(name="grad-4k", op="grad", rows=4039, V=301, F=128, dtype="f32"),
        # degree classes of the 1,130,000-node power-law graph (largest degree 29,000): a few tokens hold most rows
        dict(name="grad-1m", op="grad", rows=1_130_000, V=29_001, F=128, dtype="f32"),
        # the 10,000,000-node graph with a community-sized vocabulary, bfloat16 gradients
        dict(name="grad-10m", op="grad", rows=10_000_000, V=1_000_003, F=256, dtype="bf16"),
        # norms around a block of the 1,000-node graph, forward
        dict(name="norm-1k", op="norm", rows=1000, F=64, dtype="f32", gate="vector"),
        # a quarter of the 10,000,000-node graph (one range of subgraphs), width 256 in bfloat16, forward and backward
        dict(name="norm-2.5m", op="norm", rows=2_500_000, F=256, dtype="bf16", gate="vector"),
        dict(name="norm-bwd-2.5m", op="norm_bwd", rows=2_500_000, F=256, dtype="bf16", gate="vector"),
        # backward with a gate of its own per node, a width that no vector load divides, an odd row count
        dict(name="norm-bwd-odd", op="norm_bwd", rows=100_003, F=99, dtype="f32", gate="rows"),
        # the 1,024-subgraph model, one 128 x 128 weight per subgraph
        dict(name="muon-1024x128", op="muon", sets=1024, r=128, c=128),
        # the 4,096-subgraph model, one 256 x 256 weight per subgraph
        dict(name="muon-4096x256", op="muon", sets=4096, r=256, c=256),
        # one weight shared by all subgraphs, wide and with odd sides: a single large matrix
        dict(name="muon-shared", op="muon", sets=1, r=1000, c=1537),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "grad", "norm", "norm_bwd", "muon", "muon"])
    if op == "muon":
        if rng.random() < 0.25:
            return dict(op=op, sets=rng.randint(1, 3), r=_log_int(rng, 200, 1600), c=_log_int(rng, 200, 1600))
        r, c = _log_int(rng, 8, 256), _log_int(rng, 8, 256)
        most = 4096 * 256 ** 3 // (r * c * min(r, c))
        return dict(op=op, sets=_log_int(rng, 1, min(4096, most)), r=r, c=c)
    F, dtype = _log_int(rng, 8, 512), rng.choice(["f32", "bf16"])
    most = (2_500_000 if op.startswith("norm") else 10_000_000) * 256 * 2 // (F * (4 if dtype == "f32" else 2))
    rows = _log_int(rng, 1, min(most, 10_000_000))
    if op.startswith("norm"):
        return dict(op=op, rows=rows, F=F, dtype=dtype, gate=rng.choice(["none", "vector", "rows"]))
    return dict(op=op, rows=rows, V=_log_int(rng, 2, 1_000_003 * 256 // max(F, 256)), F=F, dtype=dtype)


def _normal(g, shape, dtype, scale=1.0, mean=0.0):
    """Standard normals in `dtype`, filled in slices so that no large float32 copy is made."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for part in out.view(-1).split(1 << 28):
        part.normal_(mean, scale, generator=g)
    return out


def _graph():
    """A handle as a user's program has one: here of a small graph, since the operators take their own sizes."""
    import paper_2511_09261_b200 as gnnco
    ids = torch.arange(8, dtype=torch.int32, device="cuda")
    return gnnco.gnnco_partition_load(ids[:-1].contiguous(), ids[1:].contiguous(), torch.zeros_like(ids), 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    if case["op"] in ("lookup", "grad"):
        rows, V, F, dtype = case["rows"], case["V"], case["F"], DTYPES[case["dtype"]]
        # token t about as 1 / (t + 1): a few classes hold most nodes; one node in a hundred has no token (-1)
        u = torch.rand(rows, device="cuda", generator=g)
        tokens = (torch.exp(u * math.log(V + 1.0)) - 1.0).to(torch.int32).clamp_(0, V - 1)
        shuffle = torch.randperm(V, device="cuda", generator=g).to(torch.int32)
        tokens = shuffle[tokens.long()]
        tokens[torch.rand(rows, device="cuda", generator=g) < 0.01] = -1
        s.update(tokens=tokens, scale=math.sqrt(F))
        if case["op"] == "lookup":
            s["table"] = _normal(g, (V, F), dtype, F ** -0.5)
        else:
            s["dout"] = _normal(g, (rows, F), dtype)
    elif case["op"] in ("norm", "norm_bwd"):
        rows, F, dtype = case["rows"], case["F"], DTYPES[case["dtype"]]
        s.update(scale=0.5, x=_normal(g, (rows, F), dtype), y=_normal(g, (rows, F), dtype, 2.0),
                 w_pre=_normal(g, (F,), torch.float32, 0.1, 1.0), w_post=_normal(g, (F,), torch.float32, 0.1, 1.0))
        s["gate"] = {"none": lambda: None, "vector": lambda: _normal(g, (F,), torch.float32, 0.3, 0.5),
                     "rows": lambda: _normal(g, (rows, F), dtype, 0.3, 0.5)}[case["gate"]]()
        if case["op"] == "norm_bwd":
            s.update(dx=_normal(g, (rows, F), dtype), dh=_normal(g, (rows, F), dtype))
    else:
        sets, r, c = case["sets"], case["r"], case["c"]
        k = min(8, r, c)
        # gradients as training has them: a few strong directions over noise
        strong = _normal(g, (sets, r, k), torch.float32) @ _normal(g, (sets, k, c), torch.float32)
        s.update(W=_normal(g, (sets, r, c), torch.float32, (2.0 / (r + c)) ** 0.5),
                 dW=strong.add_(_normal(g, (sets, r, c), torch.float32), alpha=0.5).mul_(1e-3),
                 m=_normal(g, (sets, r, c), torch.float32, 1e-3), lr=0.02, momentum=0.95, decay=0.01)
    if own:
        s["graph"] = _graph()
    return s


def _rms(x):
    return torch.rsqrt((x * x).mean(dim=1, keepdim=True) + NORM_EPS)


def _plain(s):
    op = s["op"]
    if op == "lookup":
        t = s["tokens"]
        rows = s["table"].float()[t.clamp(min=0).long()]
        return (rows * ((t >= 0).float() * s["scale"])[:, None]).to(s["table"].dtype)
    if op == "grad":
        t, V = s["tokens"], s["V"]
        d = s["dout"].float()
        acc = torch.zeros(V + 1, d.shape[1], device=d.device)
        acc.index_add_(0, torch.where(t < 0, V, t).long(), d)
        return acc[:V] * s["scale"]
    if op in ("norm", "norm_bwd"):
        dtype, scale, w1, w2 = s["x"].dtype, s["scale"], s["w_pre"], s["w_post"]
        x, y = s["x"].float(), s["y"].float()
        gate = s["gate"].float() if s["gate"] is not None else 1.0
        yhat = y * _rms(y)
        if op == "norm":
            xo = x + scale * gate * w2 * yhat
            return xo.to(dtype), (xo * _rms(xo) * w1).to(dtype)
        # x is here the residual stream after the block, as the forward pass left it
        r = _rms(x)
        xhat = x * r
        dh = s["dh"].float()
        a = dh * w1
        total = s["dx"].float() + r * (a - xhat * (a * xhat).mean(dim=1, keepdim=True))
        dw_pre = (dh * xhat).sum(dim=0)
        gt = scale * total * yhat
        b = scale * gate * w2 * total
        dy = _rms(y) * (b - yhat * (b * yhat).mean(dim=1, keepdim=True))
        out = dict(dx=total.to(dtype), dy=dy.to(dtype), dw_pre=dw_pre, dw_post=(gate * gt).sum(dim=0))
        if s["gate"] is not None:
            dg = gt * w2
            out["dgate"] = dg.sum(dim=0) if s["gate"].dim() == 1 else dg.to(dtype)
        return out
    W, m, g = s["W"], s["m"], s["dW"]
    m.mul_(s["momentum"]).add_(g)
    X = g + s["momentum"] * m
    r, c = X.shape[1:]
    if r > c:
        X = X.transpose(1, 2)
    X = X / ((X * X).sum(dim=(1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        A = X @ X.transpose(1, 2)
        X = COEFS[0] * X + (COEFS[1] * A + COEFS[2] * (A @ A)) @ X
    if r > c:
        X = X.transpose(1, 2)
    W.mul_(1.0 - s["lr"] * s["decay"]).sub_(X, alpha=s["lr"] * math.sqrt(max(1.0, c / r)))
    return W, m


def run(s):
    if not own:
        return _plain(s)
    graph, op = s["graph"], s["op"]
    if op == "lookup":
        return graph.embedding_lookup(s["table"], s["tokens"], scale=s["scale"])
    if op == "grad":
        plan = graph.embedding_plan(s["tokens"], s["V"], s["F"])      # new tokens in every pass: the ordering is timed
        return graph.embedding_grad(plan, s["dout"], scale=s["scale"])
    if op == "norm":
        return graph.block_norm(s["x"], s["w_pre"], y=s["y"], w_post=s["w_post"], gate=s["gate"], scale=s["scale"],
                                eps=NORM_EPS)
    if op == "norm_bwd":
        d = graph.block_norm_backward(s["x"], s["dh"], s["w_pre"], dx_out=s["dx"], y=s["y"], w_post=s["w_post"],
                                      gate=s["gate"], scale=s["scale"], eps=NORM_EPS)
        return {k: v for k, v in d.items() if v is not None}
    graph.muon_update(s["W"], s["m"], s["dW"], lr=s["lr"], momentum=s["momentum"], weight_decay=s["decay"],
                      steps=NS_STEPS, coefs=COEFS, eps=NS_EPS)
    return s["W"], s["m"]


def work(case):
    op = case["op"]
    if op == "muon":
        sets, r, c = case["sets"], case["r"], case["c"]
        k, n = min(r, c), max(r, c)
        # a step: X X^T (symmetric: half), its square (symmetric: half), and one full product with X
        return dict(bytes=5 * 4 * sets * r * c, flops=float(sets) * NS_STEPS * (k * k * n + k ** 3 + 2 * k * k * n))
    es = 4 if case["dtype"] == "f32" else 2
    rows, F = case["rows"], case["F"]
    if op == "lookup":
        return dict(bytes=4 * rows + min(rows, case["V"]) * F * es + rows * F * es, flops=rows * F)
    if op == "grad":
        return dict(bytes=4 * rows + rows * F * es + 4 * case["V"] * F, flops=rows * F)
    gated = case["gate"] == "rows"
    if op == "norm":
        return dict(bytes=rows * F * es * (4 + gated), flops=12 * rows * F)
    return dict(bytes=rows * F * es * (6 + 2 * gated), flops=24 * rows * F)


def _exact_norms(s, lo, hi):
    """Forward values of rows [lo, hi) in float64 with the graph that autograd differentiates."""
    leaf = lambda t: t.double().detach().requires_grad_(True)  # noqa: E731
    gate = None if s["gate"] is None else leaf(s["gate"] if s["gate"].dim() == 1 else s["gate"][lo:hi])
    x, y, w1, w2 = leaf(s["x"][lo:hi]), leaf(s["y"][lo:hi]), leaf(s["w_pre"]), leaf(s["w_post"])

    def norm(v, w):
        return v / torch.sqrt(v.pow(2).sum(1, keepdim=True) / v.shape[1] + NORM_EPS) * w

    block = norm(y, w2) * s["scale"]
    return x, y, w1, w2, gate, block if gate is None else block * gate, norm


def exact(case, seed):
    op = case["op"]
    if op == "muon" and case["sets"] * case["r"] * case["c"] * min(case["r"], case["c"]) > 1024 * 160 ** 3:
        return None                                      # over 20 s in float64
    s = prepare(case, seed)
    if op == "lookup":
        t = s["tokens"].long()
        table = torch.cat([s["table"].double() * s["scale"], torch.zeros(1, case["F"], dtype=torch.float64, device="cuda")])
        return torch.index_select(table, 0, torch.where(t < 0, case["V"], t))
    if op == "grad":
        t, V = s["tokens"].long(), case["V"]
        order = torch.argsort(t)
        ends = torch.searchsorted(t[order], torch.arange(-1, V, device="cuda"), right=True)      # rows of tokens <= t
        out = torch.empty(V, case["F"], dtype=torch.float64, device="cuda")
        for f in range(0, case["F"], 16):
            total = torch.cumsum(s["dout"][:, f:f + 16][order].double(), dim=0)
            total = torch.cat([torch.zeros_like(total[:1]), total])
            out[:, f:f + 16] = s["scale"] * (total[ends[1:]] - total[ends[:-1]])
        return out
    if op in ("norm", "norm_bwd"):
        rows, step, parts, sums = case["rows"], max(1, (1 << 26) // case["F"]), [], {}
        for lo in range(0, rows, step):
            hi = min(rows, lo + step)
            x, y, w1, w2, gate, block, norm = _exact_norms(s, lo, hi)
            if op == "norm":
                xo = x + block
                parts.append((xo.detach(), norm(xo, w1).detach()))
                continue
            # the stream x' = (x' - block) + block is the given tensor: its cotangent reaches x and the block alike
            h = norm(x, w1)
            dxn, dw1 = torch.autograd.grad(h, (x, w1), s["dh"][lo:hi].double())
            total = s["dx"][lo:hi].double() + dxn
            got = torch.autograd.grad(block, (y, w2) + (() if gate is None else (gate,)), total)
            parts.append((total, got[0]) + ((got[2],) if case["gate"] == "rows" else ()))
            for name, v in [("dw_pre", dw1), ("dw_post", got[1])] + ([("dgate", got[2])] if case["gate"] == "vector" else []):
                sums[name] = sums.get(name, 0) + v
        whole = [torch.cat(p) for p in zip(*parts)]
        if op == "norm":
            return tuple(whole)
        return {**dict(zip(("dx", "dy", "dgate"), whole)), **sums}
    m = s["momentum"] * s["m"].double() + s["dW"].double()
    u = s["dW"].double() + s["momentum"] * m
    tall = case["r"] > case["c"]
    u = u.mT if tall else u
    u = u / (torch.linalg.matrix_norm(u, keepdim=True) + NS_EPS)
    # every step multiplies from the left by a polynomial of the Gram matrix, and these all commute
    A, Q = u @ u.mT, torch.eye(u.shape[1], dtype=torch.float64, device="cuda")
    for _ in range(NS_STEPS):
        P = COEFS[0] * torch.eye(u.shape[1], dtype=torch.float64, device="cuda") + COEFS[1] * A + COEFS[2] * (A @ A)
        Q, A = P @ Q, P @ A @ P
    o = Q @ u
    step = s["lr"] * math.sqrt(max(1.0, case["c"] / case["r"]))
    return s["W"].double() * (1.0 - s["lr"] * s["decay"]) - step * (o.mT if tall else o), m
