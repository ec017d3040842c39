"""Results in the place of operands whose rows are another distance apart: one buffer, read as rows of one width and written as rows of
another.  Where a kernel reads rows while others are written such a call is refused, or another kernel takes it."""
import pytest

import paper_2511_09261_b200 as gnnco
from test_gpu_gated_ff import load, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def graph():
    return load([300, 257, 40, 0, 129] * 40)


def over(t, cols):
    """[rows, cols] of consecutive rows from the start of t's buffer."""
    return t.as_strided((t.shape[0], cols), (cols, 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,F,Fo", [(3, 64, 32), (5000, 64, 32), (5000, 32, 64), (5000, 300, 296)])
def test_forward_refuses_rows_of_another_distance(graph, dtype, rows, F, Fo):
    import torch
    x, _, *w = make(rows, 1, F, 96, Fo, dtype)
    wide = torch.zeros(rows, max(F, Fo), dtype=x.dtype, device="cuda")
    v = over(wide, F)
    v.copy_(x)
    with pytest.raises(gnnco.GnncoError) as e:
        graph.gated_ff(v, *w, out=over(wide, Fo))
    assert e.value.status == gnnco.INVALID_ARGUMENT
    torch.cuda.synchronize()
    assert torch.equal(v, x)
    # the same columns of a wide tensor, narrower or wider than what is read
    wide[:, :F] = x
    want = graph.gated_ff(x, *w)
    graph.gated_ff(wide[:, :F], *w, out=wide[:, :Fo])
    assert torch.equal(wide[:, :Fo], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("want_dw", [False, True])
@pytest.mark.parametrize("F,Fo", [(64, 128), (128, 64), (128, 40), (64, 64)])
def test_dx_over_operands(graph, dtype, want_dw, F, Fo):
    """dx in the place of dy as rows of another distance, of x with gaps, of the same rows, and in columns beside x."""
    import torch
    rows = graph.n
    x, dy, *w = make(rows, graph.S, F, 96, Fo, dtype)
    want = graph.gated_ff_backward(x, dy, *w, want_dw=want_dw)

    def check(x, dy, dx):
        d = graph.gated_ff_backward(x, dy, *w, want_dw=want_dw, dx=dx)
        torch.cuda.synchronize()
        assert all((a is None) == (d[n] is None) and (a is None or torch.equal(d[n], a)) for n, a in want.items())
    buffer = torch.zeros(rows, 2 * max(F, Fo), dtype=x.dtype, device="cuda")
    over(buffer, Fo).copy_(dy)
    check(x, over(buffer, Fo), over(buffer, F))
    buffer[:, :F] = x
    check(buffer[:, :F], dy, over(buffer, F))
    buffer[:, :F] = x
    check(buffer[:, :F], dy, buffer[:, :F])
    buffer[:, :F] = x
    check(buffer[:, :F], dy, buffer[:, F:2 * F])
    assert torch.equal(buffer[:, :F], x)
