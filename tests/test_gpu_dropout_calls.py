"""Calls of dropout at the ends of what its documentation allows."""
import numpy as np
import pytest

import ff_ref as ref
import paper_2511_09261_b200 as gnnco
from test_gpu_dropout import graph  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("F", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 31 - 4, 2 ** 31 - 8])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_row_of_two_thousand_million_elements(graph, F, dtype):  # noqa: F811
    import torch
    x = torch.ones(1, F, dtype=getattr(torch, dtype), device="cuda")
    out = graph.dropout(x, gnnco.Dropout(0.5, 42, layer=1, step=2), out=x)
    quads = -(-F // 4)
    for first in (0, quads // 2, quads - 5):
        n = np.arange(first, first + 5, dtype=np.uint64)
        counter = np.stack([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), np.full_like(n, 2), np.full_like(n, 1)], axis=1)
        words = ref.philox(counter, (42, 0)).reshape(-1)
        got = out[0, 4 * first:4 * first + 20].float().cpu().numpy()
        want = np.where(words >= np.uint64(2 ** 31), 2.0, 0.0)[:got.size]
        assert got.size >= 17 and np.array_equal(got, want), first


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_rows_of_another_distance_in_place_are_refused(graph, dtype, p):  # noqa: F811
    """A row of the result would lie over other rows of x, which other threads still read."""
    import torch
    x = torch.ones(300, 24, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    close = x.as_strided((300, 16), (16, 1))
    for a, b in ((x[:, :16], close), (close, x[:, :16])):
        with pytest.raises(gnnco.GnncoError) as e:
            graph.dropout(a, gnnco.Dropout(p, 1), out=b)
        assert e.value.status == gnnco.INVALID_ARGUMENT
    torch.cuda.synchronize()
    assert bool((x == 1).all())
    one = x[:1, :16]                                               # a single row has no distance
    assert torch.equal(graph.dropout(one, gnnco.Dropout(0.0, 1), out=close[:1]), torch.ones_like(one))
