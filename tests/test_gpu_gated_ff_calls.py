"""Calls of the block at the ends of what its documentation allows: the widest operands, very many sets of weights, a first call inside a
capture, a row that is far from the next."""
import os
import subprocess
import sys

import numpy as np
import pytest

import paper_2511_09261_b200 as gnnco
from test_gpu_gated_ff import load, make, single  # noqa: F401
from test_gpu_gated_ff_close import check

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("rows", [1, 70, 700])
@pytest.mark.parametrize("F,H,Fo", [(65536, 8, 24), (24, 65536, 8), (8, 24, 65536), (40, 40_000, 24)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_widest_operands(single, rows, F, H, Fo, dtype):  # noqa: F811
    check(single, make(rows, 1, F, H, Fo, dtype, seed=3), None, "silu", dtype, 0.1)


def test_wider_operands_are_refused(single):  # noqa: F811
    for F, H, Fo in ((65537, 8, 8), (8, 65537, 8), (8, 8, 65537)):
        t = make(2, 1, F, H, Fo, "bf16")
        for call in (lambda: single.gated_ff(t[0], *t[2:]), lambda: single.gated_ff_backward(*t)):
            with pytest.raises(gnnco.GnncoError) as e:
                call()
            assert e.value.status == gnnco.UNSUPPORTED


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_sets_than_a_grid_has_rows(dtype):
    """100,000 subgraphs of none to three nodes, against the same products in float64 row by row on the GPU."""
    import torch
    sizes = np.random.RandomState(5).randint(0, 4, 100_000)
    rows, sets, F, H = int(sizes.sum()), len(sizes), 8, 16
    g = load(sizes)
    x, dy, *w = t = make(rows, sets, F, H, F, dtype, seed=1)
    y, d = g.gated_ff(x, *w), g.gated_ff_backward(*t)
    part = torch.from_numpy(np.repeat(np.arange(sets), sizes)).cuda()
    X, D = x.double(), dy.double()
    wg, wu, wd = (v.double()[part] for v in w)
    mul = lambda a, b: torch.einsum("rk,rkn->rn", a, b)  # noqa: E731
    gate, up, dh = mul(X, wg), mul(X, wu), mul(D, wd.mT)
    s = torch.sigmoid(gate)
    h, dg, du = gate * s * up, dh * up * s * (1 + gate * (1 - s)), dh * gate * s
    want = dict(y=mul(h, wd), dx=mul(dg, wg.mT) + mul(du, wu.mT))
    for n, a, b in (("dw_gate", X, dg), ("dw_up", X, du), ("dw_down", h, D)):
        want[n] = torch.zeros(sets, a.shape[1], b.shape[1], dtype=torch.float64, device="cuda").index_add_(0, part, a[:, :, None] * b[:, None, :])
    for n, v in want.items():
        err = float(((y if n == "y" else d[n]).double() - v).norm() / v.norm())
        # float32: some thirty roundings of 2^-24 and the activation's; bfloat16: a stored operand and a result, 2^-8 / sqrt(3) each at most
        # in the mean square
        assert err < (40 * 2.0 ** -24 if dtype == "f32" else 2.0 ** -8 * (2 / 3) ** 0.5), (n, err)
    assert g.async_status() == gnnco.OK


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_first_calls_of_a_process_inside_a_capture(dtype):
    """What a first call looks up (shared memory, clusters that fit) does not break a capture."""
    program = r"""
import sys, torch
sys.path[:0] = [%r, %r]
import paper_2511_09261_b200 as gnnco
from test_gpu_gated_ff import load, make
g = load([3000, 70, 2000])
few = make(3, 1, 64, 96, 64, "f32")
t = [v.to(torch.%s) for v in make(5070, 3, 64, 96, 64, "f32")]
few = [v.to(torch.%s) for v in few]
drop = gnnco.Dropout(0.25, 3)
stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=stream):
    got = [g.gated_ff(t[0], *t[2:], drop=drop), g.gated_ff(few[0], *few[2:]), g.dropout(t[0], drop), *g.gated_ff_backward(*t, drop=drop).values()]
graph.replay()
torch.cuda.synchronize()
want = [g.gated_ff(t[0], *t[2:], drop=drop), g.gated_ff(few[0], *few[2:]), g.dropout(t[0], drop), *g.gated_ff_backward(*t, drop=drop).values()]
assert all(torch.equal(a, b) for a, b in zip(got, want)) and g.async_status() == gnnco.OK
print("equal")
""" % (ROOT, os.path.join(ROOT, "tests"), dtype, dtype)
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "equal" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_rows_far_apart(single, dtype):  # noqa: F811
    """Rows 2^31 elements apart, for x, dy and the results."""
    import torch
    ld = 1 << 31
    t = make(2, 1, 24, 40, 24, dtype)
    want, d = single.gated_ff(t[0], *t[2:]), single.gated_ff_backward(*t)
    far = torch.empty(ld + 100, dtype=t[0].dtype, device="cuda")
    x, dy, y, dx = (far.as_strided((2, 24), (ld, 1), 24 * i) for i in range(4))
    x.copy_(t[0])
    dy.copy_(t[1])
    single.gated_ff(x, *t[2:], out=y)
    e = single.gated_ff_backward(x, dy, *t[2:], dx=dx)
    assert torch.equal(y, want) and all(torch.equal(e[n], d[n]) for n in d)
