"""Timed cases of the gated feed-forward block over the subgraphs of a partition (forward and backward, one weight set per
subgraph or one for all) and of dropout whose mask is drawn from a counter-based generator and never stored.

With ``own = False`` a case runs in its plain form, elementary torch operations in float32; with ``own = True`` it runs
through the entry points of ``paper_2511_09261_b200``.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the features of the 1,000-node graph: a call of a few microseconds
        dict(name="drop-1k", op="drop", rows=1000, F=64, dtype="f32", p=0.5),
        # a width that no vector load divides, an odd row count
        dict(name="drop-odd", op="drop", rows=100_003, F=99, dtype="bf16", p=0.1),
        # a quarter of the 10,000,000-node graph (one range of subgraphs), width 256 in bfloat16
        dict(name="drop-2.5m", op="drop", rows=2_500_000, F=256, dtype="bf16", p=0.1),
        # one node evaluated again with weights that all subgraphs share: the smallest call, bound by the weights' bytes
        dict(name="ff-1", op="ff", rows=1, sets=1, F=1024, H=4096, dtype="bf16", act="silu", p=0.0),
        # the 1,000-node graph in 8 subgraphs, a block of its own for each
        dict(name="ff-1k", op="ff", rows=1000, sets=8, F=64, H=128, dtype="f32", act="silu", p=0.0),
        # the 1,130,000-node power-law graph in 1,024 subgraphs, width 128 in float32
        dict(name="ff-1.1m", op="ff", rows=1_130_000, sets=1024, F=128, H=256, dtype="f32", act="gelu", p=0.0),
        # a quarter of the 10,000,000-node graph, 1,024 subgraphs, width 256 in bfloat16, with dropout behind the block
        dict(name="ff-2.5m", op="ff", rows=2_500_000, sets=1024, F=256, H=512, dtype="bf16", act="silu", p=0.1),
        # one wide block for all nodes, an odd hidden width
        dict(name="ff-shared", op="ff", rows=65_536, sets=1, F=1024, H=2731, dtype="bf16", act="silu", p=0.0),
        # training the 1,000-node graph's blocks
        dict(name="ff-bwd-1k", op="ff_bwd", rows=1000, sets=8, F=64, H=128, dtype="f32", act="silu", p=0.0),
        # the social-ego-network shape, 16 subgraphs, an odd hidden width, float32, with dropout
        dict(name="ff-bwd-4k", op="ff_bwd", rows=4039, sets=16, F=128, H=343, dtype="f32", act="gelu", p=0.1),
        # the 1,130,000-node graph, width 128 in bfloat16
        dict(name="ff-bwd-1.1m", op="ff_bwd", rows=1_130_000, sets=1024, F=128, H=256, dtype="bf16", act="silu", p=0.1),
        # one wide block for all nodes
        dict(name="ff-bwd-shared", op="ff_bwd", rows=32_768, sets=1, F=1024, H=2816, dtype="bf16", act="silu", p=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["drop", "ff", "ff", "ff_bwd", "ff_bwd"])
    dtype = rng.choice(["f32", "bf16"])
    es = 4 if dtype == "f32" else 2
    if op == "drop":
        F = _log_int(rng, 1, 1024)
        return dict(op=op, rows=_log_int(rng, 1, min(5_000_000, 2_500_000 * 256 * 2 // (F * es))), F=F, dtype=dtype,
                    p=rng.choice([0.05, 0.1, 0.5]))
    shared = rng.random() < 0.4
    F, H = _log_int(rng, 8, 1200 if shared else 256), _log_int(rng, 8, 4096 if shared else 600)
    per_row = (6 if op == "ff" else 16) * F * H
    most = min(1_000_000_000_000 // per_row, 2_500_000, 800_000_000 // F)
    sets = 1 if shared else _log_int(rng, 2, max(2, min(1024, 400_000_000 // (F * H * es))))
    rows = _log_int(rng, 1 if shared else sets, max(most, sets))
    # (a gate next to zero lets the rectifier's gradient jump by its whole value, in any precision: it is drawn forward only)
    acts = ["silu", "gelu", "relu"] if op == "ff" else ["silu", "gelu"]
    return dict(op=op, rows=rows, sets=sets, F=F, H=H, dtype=dtype, act=rng.choice(acts), p=rng.choice([0.0, 0.1]))


def _normal(g, shape, dtype, scale=1.0):
    """Normals in `dtype`, filled in slices so that no large float32 copy is made."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for part in out.view(-1).split(1 << 28):
        part.normal_(0.0, scale, generator=g)
    return out


def _graph(part, sets):
    """A handle as a user's program has one, for nodes that are sorted by subgraph already."""
    import paper_2511_09261_b200 as gnnco
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    return gnnco.gnnco_partition_load(none, none, part, sets)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    rows, F, dtype = case["rows"], case["F"], DTYPES[case["dtype"]]
    s.update(x=_normal(g, (rows, F), dtype), drop_seed=(int(seed) * 7919 + 12345) * 0x10001000101 % 2 ** 63, layer=3, step=int(seed) % 1000)
    part, sets = torch.zeros(rows, dtype=torch.int32, device="cuda"), 1
    if case["op"] != "drop":
        sets, H = case["sets"], case["H"]
        s.update(w_gate=_normal(g, (sets, F, H), dtype, F ** -0.5), w_up=_normal(g, (sets, F, H), dtype, F ** -0.5),
                 w_down=_normal(g, (sets, H, F), dtype, H ** -0.5))
        if sets > 1:
            # subgraphs of about equal size, as breadth-first growth leaves them, the last ones smaller or empty
            share = torch.rand(sets, device="cuda", generator=g) * 0.2 + 0.9
            ends = (torch.cumsum(share.double(), 0) / share.double().sum() * rows).round().long()
            part = torch.searchsorted(ends, torch.arange(rows, device="cuda"), right=True).clamp_(max=sets - 1).int()
        if case["op"] == "ff_bwd":
            s["dy"] = _normal(g, (rows, F), dtype)
    counts = torch.bincount(part.long(), minlength=sets)
    first = torch.cumsum(counts, 0) - counts
    # where every node's row stands in its subgraph: a program of such blocks keeps it beside the partition
    s.update(set_of=part.long(), place=torch.arange(rows, device="cuda") - first[part.long()], longest=int(counts.max()))
    if own:
        import paper_2511_09261_b200 as gnnco
        s["graph"] = _graph(part, sets)
        s["drop"] = gnnco.Dropout(case["p"], s["drop_seed"], layer=s["layer"], step=s["step"]) if case["p"] else None
    return s


def _words(s, rows, F):
    """32-bit words of Philox4x32-10, one per element: element (r, c) takes word c % 4 of counter
    (r * ceil(F / 4) + c // 4, step, layer) under the seed."""
    low = 0xFFFFFFFF
    quads = -(-F // 4)
    q = torch.arange(rows * quads, device="cuda")
    c0, c1 = q & low, q >> 32
    c2, c3 = torch.full_like(q, s["step"]), torch.full_like(q, s["layer"])
    k0, k1 = s["drop_seed"] & low, s["drop_seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                       # the upper half survives the wrap of 64 bits
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), dim=1).view(rows, quads * 4)[:, :F]


def _drop(s, x):
    """x float32: elements whose word is below p * 2^32 become 0, the others are scaled by 1 / (1 - p)."""
    if not s["p"]:
        return x
    keep = _words(s, *x.shape) >= round(s["p"] * 2.0 ** 32)
    return torch.where(keep, x * (1.0 / (1.0 - s["p"])), torch.zeros_like(x))


def _act(name, g):
    """The activation and its derivative."""
    if name == "relu":
        on = (g > 0).float()
        return g * on, on
    if name == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _by_set(s, t):
    """[rows, F] -> [sets, longest subgraph, F] with rows of zeros behind the shorter ones."""
    if s["sets"] == 1:
        return t[None]
    out = torch.zeros(s["sets"], s["longest"], t.shape[1], device=t.device)
    out[s["set_of"], s["place"]] = t
    return out


def _by_row(s, t):
    return t[0] if s["sets"] == 1 else t[s["set_of"], s["place"]]


def _plain(s):
    dtype = s["x"].dtype
    if s["op"] == "drop":
        return _drop(s, s["x"].float()).to(dtype)
    wg, wu, wd = s["w_gate"].float(), s["w_up"].float(), s["w_down"].float()
    x = _by_set(s, s["x"].float())
    gate, up = torch.matmul(x, wg), torch.matmul(x, wu)
    a, slope = _act(s["act"], gate)
    if s["op"] == "ff":
        return _drop(s, _by_row(s, torch.matmul(a * up, wd))).to(dtype)
    dy = _by_set(s, _drop(s, s["dy"].float()))
    dh = torch.matmul(dy, wd.mT)
    dw_down = torch.matmul((a * up).mT, dy)
    dgate, dup = dh * up * slope, dh * a
    dx = torch.matmul(dgate, wg.mT) + torch.matmul(dup, wu.mT)
    return dict(dx=_by_row(s, dx).to(dtype), dw_gate=torch.matmul(x.mT, dgate).to(dtype),
                dw_up=torch.matmul(x.mT, dup).to(dtype), dw_down=dw_down.to(dtype))


def run(s):
    if not own:
        return _plain(s)
    graph = s["graph"]
    if s["op"] == "drop":
        return graph.dropout(s["x"], s["drop"])
    if s["op"] == "ff":
        return graph.gated_ff(s["x"], s["w_gate"], s["w_up"], s["w_down"], act=s["act"], drop=s["drop"])
    return graph.gated_ff_backward(s["x"], s["dy"], s["w_gate"], s["w_up"], s["w_down"], act=s["act"], drop=s["drop"])


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    rows, F = case["rows"], case["F"]
    if case["op"] == "drop":
        return dict(bytes=2 * rows * F * es, flops=2 * rows * F)
    H = case["H"]
    weights = 3 * min(case["sets"], rows) * F * H * es
    if case["op"] == "ff":
        return dict(bytes=2 * rows * F * es + weights, flops=6.0 * rows * F * H)
    # gate and up again, then dh, dx (two products) and three weight gradients
    return dict(bytes=3 * rows * F * es + weights + 3 * case["sets"] * F * H * es, flops=16.0 * rows * F * H)


def _keep(s, rows, F):
    """The kept elements, from the generator's definition with 16-bit halves: no product leaves 53 bits."""
    def split_product(m, v):
        mh, ml, vh, vl = m >> 16, m & 0xFFFF, v // 65536, v % 65536
        middle = mh * vl + (ml * vl) // 65536
        cross = ml * vh + middle % 65536
        return mh * vh + middle // 65536 + cross // 65536, (cross % 65536) * 65536 + (ml * vl) % 65536

    quads = (F + 3) // 4
    out = torch.empty(rows, quads, 4, dtype=torch.bool, device="cuda")
    limit = round(s["p"] * 2.0 ** 32)
    for lo in range(0, rows, 1 << 18):
        hi = min(rows, lo + (1 << 18))
        n = torch.arange(lo * quads, hi * quads, device="cuda").reshape(hi - lo, quads)
        c = [n % 2 ** 32, n // 2 ** 32, torch.full_like(n, s["step"]), torch.full_like(n, s["layer"])]
        key = [s["drop_seed"] % 2 ** 32, s["drop_seed"] // 2 ** 32]
        for _ in range(10):
            h0, l0 = split_product(0xD2511F53, c[0])
            h1, l1 = split_product(0xCD9E8D57, c[2])
            c = [h1.bitwise_xor(c[1]).bitwise_xor(key[0]), l1, h0.bitwise_xor(c[3]).bitwise_xor(key[1]), l0]
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        for k in range(4):
            out[lo:hi, :, k] = c[k] >= limit
    return out.reshape(rows, quads * 4)[:, :F]


_EXACT_ACT = {"relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
              "gelu": lambda v: v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))}


def exact(case, seed):
    s = prepare(case, seed)
    rows, F = case["rows"], case["F"]
    mask = _keep(s, rows, F).double() / (1.0 - case["p"]) if case["p"] else None
    if case["op"] == "drop":
        return s["x"].double() * mask
    sizes = torch.bincount(s["set_of"], minlength=case["sets"]).tolist()
    outs, grads, lo = [], [], 0
    for k, size in enumerate(sizes):
        w = [s[n][k].double().requires_grad_(True) for n in ("w_gate", "w_up", "w_down")]
        total = [torch.zeros_like(v) for v in w]
        # slices of rows, so that one set's tensors in 64 bits stay small
        for a in range(lo, lo + size, 16384):
            b = min(lo + size, a + 16384)
            x = s["x"][a:b].double().requires_grad_(True)
            y = (_EXACT_ACT[case["act"]](x @ w[0]) * (x @ w[1])) @ w[2]
            if mask is not None:
                y = y * mask[a:b]
            if case["op"] == "ff":
                outs.append(y.detach())
                continue
            got = torch.autograd.grad(y, [x] + w, s["dy"][a:b].double())
            outs.append(got[0])
            total = [t + d for t, d in zip(total, got[1:])]
        lo += size
        grads.append(total)
    out = torch.cat(outs)
    if case["op"] == "ff":
        return out
    return dict(dx=out, **{n: torch.stack([t[i] for t in grads]).detach() for i, n in enumerate(("dw_gate", "dw_up", "dw_down"))})
