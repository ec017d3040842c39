"""The block on the GPU against float64 by the bounds of ff_close, which wrong remainders, limbs and derivatives do not pass at any of these
sizes (test_ff_close.py), and with the rectifier on whole numbers, bit by bit, over every kernel that the block may go to."""
import numpy as np
import pytest

import ff_close as close
import ff_ref as ref
import paper_2511_09261_b200 as gnnco
from test_gpu_gated_ff import FEW, SHAPES, dev, host, load, make, single  # noqa: F401

pytestmark = pytest.mark.gpu

MANY = [300, 0, 257, 1, 33, 5000, 256] * 6 + [640] * 10


def ptr_of(sizes):
    return np.concatenate([[0], np.cumsum(sizes)])


def check(g, t, ptr, act, dtype, p=0.0, forward=True, back=True, **k):
    """The largest part of what is allowed, for every result."""
    x, dy, *w = t
    rows, F, H, Fo = x.shape[0], x.shape[1], w[0].shape[2], w[2].shape[2]
    drop = gnnco.Dropout(p, 21, layer=2, step=3) if p else None
    mask = ref.keep(rows, Fo, p, 21, 2, 3) / (1 - p) if p else None
    # float32 weights of bfloat16 features are rounded to bfloat16
    hx, hdy, *hw = [host(t[i]) for i in (0, 1)] + [host(v.bfloat16() if dtype == "bf16" else v) for v in w]
    longest = int(np.diff(ptr).max()) if ptr is not None and w[0].shape[0] > 1 else rows
    r = {}
    if forward:
        y = g.gated_ff(x, *w, act=act, drop=drop)
        r["y"] = close.worst(host(y), close.forward(hx, *hw, ptr, act, mask), dtype, F, H, dtype == "bf16")
    if back:
        d = g.gated_ff_backward(x, dy, *w, act=act, drop=drop, **k)
        for n, want in close.backward(hx, hdy, *hw, ptr, act, mask).items():
            sets = n[:2] == "dw"
            r[n] = close.worst(host(d[n]), want, dtype, max(F, Fo), longest if sets else 2 * H, d[n].element_size() == 2, 0 if sets else None)
    assert max(r.values()) <= 1.0, r
    assert g.async_status() == gnnco.OK


@pytest.mark.parametrize("rows,F,H,Fo", SHAPES + [(33, 1000, 2100, 300), (20_011, 72, 521, 257)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,p", [("silu", 0.0), ("gelu", 0.3)])
def test_one_set(single, rows, F, H, Fo, dtype, act, p):  # noqa: F811
    check(single, make(rows, 1, F, H, Fo, dtype, seed=7), None, act, dtype, p)


@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("F,H,Fo", [(40, 56, 24), (1024, 4096, 1024), (99, 343, 51), (64, 3000, 8), (5000, 33, 16)])
@pytest.mark.parametrize("dtype,w_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_few_rows(single, rows, F, H, Fo, dtype, w_dtype, act):  # noqa: F811
    check(single, make(rows, 1, F, H, Fo, dtype, seed=rows, w_dtype=w_dtype), None, act, dtype, back=False)


@pytest.mark.parametrize("sizes", [FEW, MANY, [125] * 8, [0, 2500, 10], [70_000, 1, 2050]], ids=["few", "many", "even", "long", "split"])
@pytest.mark.parametrize("F,H,Fo", [(64, 128, 64), (33, 72, 21), (128, 256, 128), (200, 300, 264)])
@pytest.mark.parametrize("dtype,w_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_a_set_per_subgraph(sizes, F, H, Fo, dtype, w_dtype):
    ptr = ptr_of(sizes)
    act, p = (("silu", 0.1), ("gelu", 0.0))[(F + len(sizes)) % 2]
    check(load(sizes), make(int(ptr[-1]), len(sizes), F, H, Fo, dtype, seed=F, w_dtype=w_dtype), ptr, act, dtype, p)


# What decides between the kernels: rows (up to four; tiles enough for pairs of CTAs or not), subgraphs and how few rows they have, widths
# (128, 256: one kernel in bfloat16), the length of H
WHOLE = [
    ([1], 1, 24, 40, 16), ([2], 1, 99, 343, 51), ([3], 1, 1024, 4096, 512), ([4], 1, 64, 3000, 8),
    ([5], 1, 24, 40, 16), ([130], 1, 99, 343, 51), ([300], 1, 300, 72, 264), ([7000], 1, 130, 521, 257), ([20_011], 1, 72, 1100, 300),
    ([9_001], 1, 96, 300, 40), ([40_000], 1, 128, 256, 128), ([70_001], 1, 20, 24, 20),
    (FEW, 0, 33, 65, 21), (FEW, 0, 384, 1024, 384), (FEW, 0, 8, 8, 400),
    (MANY, 0, 16, 200, 16), (MANY, 0, 128, 256, 128), (MANY, 0, 33, 130, 65), (MANY, 0, 256, 512, 200), (MANY, 0, 264, 300, 272),
    ([70_000, 1, 0, 2050], 0, 40, 136, 24),
]


@pytest.mark.parametrize("sizes,sets,F,H,Fo", WHOLE, ids=["-".join(map(str, (sum(w[0]), w[1] or len(w[0])) + w[2:])) for w in WHOLE])
@pytest.mark.parametrize("dtype,w_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_the_rectifier_on_whole_numbers_is_exact(sizes, sets, F, H, Fo, dtype, w_dtype, p):
    import torch
    g, ptr, rows = load(sizes), ptr_of(sizes), sum(sizes)
    t = close.whole_numbers(rows, sets or len(sizes), F, H, Fo, seed=H)
    x, dy, *w = [dev(v, dtype if i < 2 else w_dtype) for i, v in enumerate(t)]
    drop = gnnco.Dropout(p, 9, layer=1, step=4) if p else None
    mask = ref.keep(rows, Fo, p, 9, 1, 4) * 2.0 if p else None
    feat, weight = x.dtype, w[0].dtype
    want = torch.from_numpy(ref.gated_ff(*t[:1], *t[2:], ptr, "relu", mask)[0]).to(feat)
    assert torch.equal(g.gated_ff(x, *w, act="relu", drop=drop).cpu(), want)
    back = ref.gated_ff_backward(*t, ptr, "relu", mask)
    want = {n: torch.from_numpy(back[n]).to(feat if n == "dx" else weight) for n in ("dx", "dw_gate", "dw_up", "dw_down")}
    d = g.gated_ff_backward(x, dy, *w, act="relu", drop=drop)
    assert all(torch.equal(d[n].cpu(), v) for n, v in want.items()), [n for n, v in want.items() if not torch.equal(d[n].cpu(), v)]
    only = g.gated_ff_backward(x, dy, *w, act="relu", drop=drop, want_dw=False)["dx"]
    assert torch.equal(only, d["dx"])
    only = g.gated_ff_backward(x, dy, *w, act="relu", drop=drop, want_dx=False)
    assert all(torch.equal(only[n], d[n]) for n in want if n != "dx")
    assert g.async_status() == gnnco.OK
