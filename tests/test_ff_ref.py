"""The float64 restatements of dropout and the gated feed-forward block, checked by themselves: published generator vectors,
moments of the mask, differences of the gradients.  And what the binding of dropout refuses, without a GPU."""
import numpy as np
import pytest
import torch

import ff_ref as ref
import paper_2511_09261_b200 as gnnco
from test_operator_calls import _Library


# known answers of Philox4x32-10 from the generator's authors
VECTORS = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


@pytest.mark.parametrize("counter,key,want", VECTORS)
def test_philox_known_answers(counter, key, want):
    got = ref.philox(np.array([counter], dtype=np.uint64), key)
    assert tuple(int(v) for v in got[0]) == want


def test_masks_keep_the_right_share_and_differ():
    a = ref.keep(400, 250, 0.3, seed=5)
    # 100,000 independent draws: five standard deviations are 0.0073
    assert abs(a.mean() - 0.7) < 0.0073
    for other in (ref.keep(400, 250, 0.3, seed=6), ref.keep(400, 250, 0.3, 5, layer=1), ref.keep(400, 250, 0.3, 5, step=1),
                  ref.keep(400, 250, 0.3, 5 + (1 << 32))):
        # independent masks agree with probability 0.58
        assert abs((a == other).mean() - 0.58) < 0.0079
    assert np.array_equal(ref.keep(10, 250, 0.3, 5, row0=390), a[390:])
    assert ref.keep(3, 5, 0.0, 5).all() and not ref.keep(3, 5, 1.0, 5).any()


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_block_gradients_against_differences(name):
    r = np.random.RandomState(3)
    ptr, F, H = [0, 4, 4, 7], 5, 6
    x, dy = r.standard_normal((7, F)), r.standard_normal((7, 4))
    w = [r.standard_normal(s) for s in ((3, F, H), (3, F, H), (3, H, 4))]
    mask = ref.keep(7, 4, 0.4, 9) / 0.6
    d = ref.gated_ff_backward(x, dy, *w, ptr, name, mask)

    def loss():
        return float((ref.gated_ff(x, *w, ptr, name, mask)[0] * dy).sum())

    for t, key in [(x, "dx"), (w[0], "dw_gate"), (w[1], "dw_up"), (w[2], "dw_down")]:
        got = np.zeros_like(t)
        for i in np.ndindex(t.shape):
            keep, eps = t[i], 1e-6
            t[i] = keep + eps
            up = loss()
            t[i] = keep - eps
            got[i] = (up - loss()) / (2 * eps)
            t[i] = keep
        np.testing.assert_allclose(got, d[key], rtol=2e-6, atol=2e-8)
        assert np.all(d[key + "_stored"] * (1 + 1e-12) >= np.abs(d[key])) and np.all(d[key + "_mag"] >= d[key + "_stored"])


@pytest.fixture
def graph(monkeypatch):
    g = gnnco.PartitionedGraph.__new__(gnnco.PartitionedGraph)
    g._lib, g._handle, g.device = _Library(), None, torch.device("cpu")
    monkeypatch.setattr(gnnco, "_stream_ptr", lambda stream=None: 0)
    return g


@pytest.mark.parametrize("drop", [
    gnnco.Dropout(-0.1, 1), gnnco.Dropout(1.5, 1), gnnco.Dropout(float("nan"), 1), gnnco.Dropout(0.1, 1 << 64),
    gnnco.Dropout(0.1, -1), gnnco.Dropout(0.1, 1, layer=1 << 32), gnnco.Dropout(0.1, 1, step=-1),
])
def test_dropout_refuses_what_the_generator_cannot_take(graph, drop):
    with pytest.raises(ValueError):
        graph.dropout(torch.ones(3, 4), drop)
    assert not graph._lib.calls


def test_dropout_refuses_other_shapes_types_and_devices(graph):
    drop, x = gnnco.Dropout(0.1, 1), torch.ones(6, 4)
    for bad in (torch.ones(4), torch.ones(2, 3, 4), torch.ones(3, 0)):
        with pytest.raises(ValueError):
            graph.dropout(bad, drop)
    for bad in (x.double(), x.half(), x.int()):
        with pytest.raises(TypeError):
            graph.dropout(bad, drop)
    for bad in (x.t(), x[:, ::2], x[:1].expand(6, 4)):
        with pytest.raises(ValueError):
            graph.dropout(bad, drop)
    for bad in (torch.empty(6, 5), torch.empty(5, 4)):
        with pytest.raises(ValueError):
            graph.dropout(x, drop, out=bad)
    with pytest.raises(TypeError):
        graph.dropout(x, drop, out=torch.empty(6, 4, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        graph.dropout(x, gnnco.Dropout(0.1, 1, step_dev=torch.zeros(1, dtype=torch.int64)))
    assert not graph._lib.calls
    graph.dropout(x[:, 1:3], drop)
    assert graph._lib.last("gnnco_dropout")[5] == 4


def _block(rows=6, F=4, H=5, Fo=3, sets=1):
    return [torch.ones(rows, F), torch.ones(sets, F, H), torch.ones(sets, F, H), torch.ones(sets, H, Fo)]


def test_block_refuses_other_shapes_and_types(graph, monkeypatch):
    monkeypatch.setattr(gnnco, "_require", _require_on_cpu)
    graph.S, graph.n = 3, 6
    bf = torch.bfloat16
    for change, error in [
        ({0: torch.ones(6)}, ValueError), ({0: torch.ones(6, 5)}, ValueError), ({0: torch.ones(6, 8)[:, ::2]}, ValueError),
        ({1: torch.ones(1, 4, 6)}, ValueError), ({2: torch.ones(1, 5, 5)}, ValueError), ({3: torch.ones(1, 4, 3)}, ValueError),
        ({1: torch.ones(4, 5)}, ValueError), ({1: torch.ones(2, 4, 5), 2: torch.ones(2, 4, 5), 3: torch.ones(2, 5, 3)}, ValueError),
        ({2: torch.ones(3, 4, 5)}, ValueError), ({3: torch.ones(1, 5, 0)}, ValueError), ({1: torch.ones(1, 5, 4).mT}, TypeError),
        ({0: torch.ones(6, 4).double()}, TypeError), ({1: torch.ones(1, 4, 5).half()}, TypeError), ({3: torch.ones(1, 5, 3, dtype=bf)}, TypeError),
    ]:
        args = [change.get(i, t) for i, t in enumerate(_block())]
        with pytest.raises(error):
            graph.gated_ff(*args)
        with pytest.raises(error):
            graph.gated_ff_backward(args[0], torch.ones(6, 3), *args[1:])
    args = _block()
    with pytest.raises(ValueError):
        graph.gated_ff(*args, act="tanh")
    with pytest.raises(ValueError):
        graph.gated_ff(*args, drop=gnnco.Dropout(2.0, 1))
    with pytest.raises(ValueError):
        graph.gated_ff(*args, out=torch.empty(6, 4))
    for dy in (torch.ones(5, 3), torch.ones(6, 4)):
        with pytest.raises(ValueError):
            graph.gated_ff_backward(args[0], dy, *args[1:])
    with pytest.raises(TypeError):
        graph.gated_ff_backward(args[0], torch.ones(6, 3, dtype=bf), *args[1:])
    with pytest.raises(TypeError):
        graph.gated_ff_backward(args[0], torch.ones(6, 3), *args[1:], dw_dtype=torch.float16)
    with pytest.raises(ValueError):
        graph.gated_ff_backward(args[0], torch.ones(6, 3), *args[1:], want_dx=False, want_dw=False)
    assert not [c for c in graph._lib.calls if not c[0].endswith("_bytes")]


def _require_on_cpu(t, dtype, what, device_type="cuda", real=gnnco._require):
    return real(t, dtype, what, "cpu")


def test_block_gradients_take_the_types_asked_for(graph, monkeypatch):
    monkeypatch.setattr(gnnco, "_require", _require_on_cpu)
    x, *w = _block()
    xb, wb = x.bfloat16(), [t.bfloat16() for t in w]
    dy = torch.ones(6, 3)
    assert graph.gated_ff_backward(x, dy, *w)["dw_up"].dtype == torch.float32
    assert graph.gated_ff_backward(xb, dy.bfloat16(), *wb)["dw_up"].dtype == torch.bfloat16
    assert graph.gated_ff_backward(xb, dy.bfloat16(), *wb, dw_dtype=torch.float32)["dw_up"].dtype == torch.float32
    d = graph.gated_ff_backward(xb, dy.bfloat16(), *w, want_dx=False)
    assert d["dx"] is None and d["dw_down"].dtype == torch.float32
    assert graph.gated_ff_backward(x, dy, *w, want_dw=False)["dw_gate"] is None


def test_the_c_entry_checks_its_arguments_without_a_gpu():
    import ctypes
    lib = gnnco.load_library()
    d = gnnco.DropoutParams(0.5, 1, 0, 0, None)
    f = gnnco.GatedFfDesc(1, 1, 1, 1, 0, 0, 1, 0)
    n = ctypes.c_size_t(0)
    assert lib.gnnco_gated_ff_workspace_bytes(None, ctypes.byref(f), 0, ctypes.byref(n)) == gnnco.INVALID_ARGUMENT
    assert lib.gnnco_gated_ff(None, ctypes.byref(f), None, 1, None, 0, None) == gnnco.INVALID_ARGUMENT
    assert lib.gnnco_gated_ff_backward(None, ctypes.byref(f), None, 1, None, None, 0, None) == gnnco.INVALID_ARGUMENT
    assert lib.gnnco_dropout(None, 0, 1, 1, None, 1, ctypes.byref(d), None, 1, None) == gnnco.INVALID_ARGUMENT
