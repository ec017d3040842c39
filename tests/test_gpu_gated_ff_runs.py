"""Weight gradients of subgraphs so long that their runs of rows are cut at 65,536: 45 M nodes would have runs of 76,032 on 148 SMs."""
import pytest

import paper_2511_09261_b200 as gnnco

pytestmark = pytest.mark.gpu


def test_subgraphs_of_many_million_rows():
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    sizes, F, H = [30_000_000, 0, 65_537, 14_900_000, 12], 8, 8
    rows, sets = sum(sizes), len(sizes)
    part = torch.repeat_interleave(torch.arange(sets, dtype=torch.int32, device="cuda"), torch.tensor(sizes, device="cuda"))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    g = gnnco.gnnco_partition_load(none, none, part, sets)
    r = torch.Generator(device="cuda").manual_seed(8)
    # gradients around one, so that the sums grow with the rows and what is cut off does not cancel
    x = torch.empty(rows, F, dtype=torch.bfloat16, device="cuda").normal_(1.0, 0.25, generator=r)
    dy = torch.empty(rows, F, dtype=torch.bfloat16, device="cuda").normal_(1.0, 0.25, generator=r)
    w = [torch.empty(s, dtype=torch.bfloat16, device="cuda").uniform_(0.05, 0.25, generator=r) for s in ((sets, F, H), (sets, F, H), (sets, H, F))]
    d = g.gated_ff_backward(x, dy, *w, want_dx=False, dw_dtype=torch.float32)
    again = g.gated_ff_backward(x, dy, *w, want_dx=False, dw_dtype=torch.float32)
    lo = 0
    for s, size in enumerate(sizes):
        wg, wu, wd = (v[s].double() for v in w)
        want = [torch.zeros(F, H, dtype=torch.float64, device="cuda"), torch.zeros(F, H, dtype=torch.float64, device="cuda"),
                torch.zeros(H, F, dtype=torch.float64, device="cuda")]
        for a in range(lo, lo + size, 1 << 20):
            b = min(lo + size, a + (1 << 20))
            xs, ds = x[a:b].double(), dy[a:b].double()
            gate, up, dh = xs @ wg, xs @ wu, ds @ wd.T
            sig = torch.sigmoid(gate)
            want[0] += xs.T @ (dh * up * sig * (1 + gate * (1 - sig)))
            want[1] += xs.T @ (dh * gate * sig)
            want[2] += (gate * sig * up).T @ ds
        lo += size
        for n, v in zip(("dw_gate", "dw_up", "dw_down"), want):
            assert torch.equal(d[n][s], again[n][s])
            if size == 0:
                assert not d[n][s].any()
                continue
            # terms of one sign: 65,536 rows in one sum lose 65,536 x 2^-27 of it at most; the roundings of the stored operand (2^-8 each)
            # and of the joined runs (2^-24 each, 458 of them) average out but for the few rows of the last subgraph
            err = float(((d[n][s].double() - v) / v).abs().max())
            assert err <= 65536 * 2.0 ** -27 + (2.0 ** -8 if size < 1000 else 2.0 ** -13), (n, s, err)
    assert g.async_status() == gnnco.OK
