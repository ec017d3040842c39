"""The gated feed-forward block on the GPU, forward and backward, against the float64 restatement."""
import numpy as np
import pytest

import ff_ref as ref
import paper_2511_09261_b200 as gnnco

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = 2.0 ** -8                # half a step of bfloat16, relative


def load(sizes):
    """A handle for subgraphs of the given numbers of nodes, nodes in order."""
    import torch
    part = torch.from_numpy(np.repeat(np.arange(len(sizes)), sizes).astype(np.int32)).cuda()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    return gnnco.gnnco_partition_load(none, none, part, len(sizes))


@pytest.fixture(scope="module")
def single():
    return load([5, 3])


def dev(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def host(t):
    return t.double().cpu().numpy()


def make(rows, sets, F, H, Fo, dtype, seed=0, w_dtype=None, whole=False):
    """x, dy, wg, wu, wd on the GPU; whole: small integers, with which every product and sum is exact."""
    r = np.random.RandomState(seed)

    def draw(scale, *shape):
        return r.randint(-2, 3, shape) if whole else r.standard_normal(shape) * scale
    w_dtype = w_dtype or dtype
    return (dev(draw(1.0, rows, F), dtype), dev(draw(1.0, rows, Fo), dtype), dev(draw(F ** -0.5, sets, F, H), w_dtype),
            dev(draw(F ** -0.5, sets, F, H), w_dtype), dev(draw(H ** -0.5, sets, H, Fo), w_dtype))


def roundings(K):
    """Units of 2^-24 of the sizes of the terms that a sum over K is off by at most.  float32 operands: what the three limbs leave
    out (1); a stage of 64 adds 24 products of 16 terms, the 4 large ones each cut off by at most 2^-23 where terms are aligned and
    again where they are added to the sum (16), the 20 small ones 2^-8 of that (1); the stages are added in float32, K / 64
    roundings.  bfloat16 operands: products are exact, K / 16 additions are cut off by 2^-23, twice each."""
    return 18 + K / 64, 4 + K / 4


def close(got, want, mag, stored, dtype, units, out_bf16):
    """`units` roundings of float32 on the terms; in bfloat16 features the stored h, dg, du are rounded (BF), after the fast forms of
    the activation (2^-20 of the terms), and a bfloat16 result once more."""
    got = host(got)
    assert got.shape == want.shape and np.all(np.isfinite(got))
    bound = units * U * mag + 1e-35
    if dtype == "bf16":
        bound = bound + BF * (1 + BF) * stored + 2.0 ** -20 * mag
    if out_bf16:
        bound = bound + BF * (np.abs(want) + bound)
    worst = float((np.abs(got - want) / bound).max()) if got.size else 0.0
    assert worst <= 1.0, worst


def check_forward(g, t, ptr, act, dtype, drop=None, mask=None, **k):
    x, _, wg, wu, wd = t
    y = g.gated_ff(x, wg, wu, wd, act=act, drop=drop, **k)
    # float32 weights of bfloat16 features are rounded to bfloat16
    w = [host(v.bfloat16() if dtype == "bf16" else v) for v in (wg, wu, wd)]
    want, mag, stored = ref.gated_ff(host(x), *w, ptr, act, mask)
    i = 1 if dtype == "bf16" else 0
    # g and u each carry their sum's error into h (1.13 for the slope of the activation), h a few roundings, then y's sum
    units = 2.3 * roundings(x.shape[1])[i] + 12 + roundings(wg.shape[2])[i] + (4 if mask is not None else 0)
    close(y, want, mag, stored, dtype, units, dtype == "bf16")
    return y


def check_backward(g, t, ptr, act, dtype, drop=None, mask=None, slots=0, **k):
    x, dy, wg, wu, wd = t
    d = g.gated_ff_backward(x, dy, wg, wu, wd, act=act, drop=drop, **k)
    w = [host(v.bfloat16() if dtype == "bf16" else v) for v in (wg, wu, wd)]
    want = ref.gated_ff_backward(host(x), host(dy), *w, ptr, act, mask)
    i = 1 if dtype == "bf16" else 0
    F, H, Fo, rows = x.shape[1], wg.shape[2], wd.shape[2], x.shape[0]
    # dh, u and the slope each carry their sum's error into dg
    inner = roundings(Fo)[i] + 3 * roundings(F)[i] + 16 + (4 if mask is not None else 0)
    for name in ("dx", "dw_gate", "dw_up", "dw_down"):
        if d[name] is None:
            continue
        outer = 2 * roundings(H)[i] if name == "dx" else roundings(rows)[i] + slots
        close(d[name], want[name], want[name + "_mag"], want[name + "_stored"], dtype, inner + outer, d[name].element_size() == 2)
    return d


# rows, F, H, F_out: one set.  Single CTAs and pairs, one stage and many, widths on both sides of tiles and vectors
SHAPES = [(1, 1, 1, 1), (1, 8, 8, 8), (3, 5, 7, 2), (2, 64, 128, 64), (9, 16, 24, 40), (127, 64, 64, 64), (128, 65, 33, 17),
          (129, 100, 96, 100), (300, 128, 200, 128), (257, 256, 512, 256), (1000, 99, 343, 99), (40, 1000, 72, 264), (65, 24, 1000, 8),
          (5000, 128, 300, 128), (4800, 264, 640, 200), (7000, 130, 521, 257)]


@pytest.mark.parametrize("rows,F,H,Fo", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(single, rows, F, H, Fo, dtype):
    act = ("silu", "gelu")[(rows + H) % 2]
    check_forward(single, make(rows, 1, F, H, Fo, dtype), None, act, dtype)


@pytest.mark.parametrize("rows,F,H,Fo", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(single, rows, F, H, Fo, dtype):
    act = ("silu", "gelu")[(rows + H + 1) % 2]
    check_backward(single, make(rows, 1, F, H, Fo, dtype), None, act, dtype, slots=16)


SIZES = [[125] * 8, [1, 0, 3, 130, 128, 0], [300, 64, 63, 65, 1], [0, 2500, 10], list(range(0, 90))]


@pytest.mark.parametrize("k", range(len(SIZES)))
@pytest.mark.parametrize("F,H,Fo", [(64, 128, 64), (40, 72, 24), (33, 19, 21), (128, 256, 128)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_set_per_subgraph(k, F, H, Fo, dtype):
    sizes = SIZES[k]
    ptr = np.concatenate([[0], np.cumsum(sizes)])
    g = load(sizes)
    t = make(int(ptr[-1]), len(sizes), F, H, Fo, dtype, seed=k)
    check_forward(g, t, ptr, "silu", dtype)
    d = check_backward(g, t, ptr, "gelu", dtype, slots=16)
    for s, size in enumerate(sizes):
        if size == 0:
            assert not any(d[n][s].any() for n in ("dw_gate", "dw_up", "dw_down"))
    assert g.async_status() == gnnco.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_whole_numbers_are_exact(single, dtype):
    """Small integers and the rectifier: every product and sum is exact, at its kink too (a gate of exactly zero passes nothing
    back)."""
    t = make(200, 1, 5, 24, 16, dtype, whole=True)
    x, dy, wg, wu, wd = t
    h = [host(v) for v in t]
    want = ref.gated_ff(h[0], h[2], h[3], h[4], None, "relu")[0]
    got = host(single.gated_ff(x, wg, wu, wd, act="relu"))
    back = ref.gated_ff_backward(*h, None, "relu")
    d = single.gated_ff_backward(x, dy, wg, wu, wd, act="relu")
    if dtype == "f32":
        assert np.array_equal(got, want)
        for n in d:
            assert np.array_equal(host(d[n]), back[n]), n
    else:
        # h and dg are at most 20 * 20 and 64 * 20: stored with 8 bits, one rounding each, one for the result
        assert np.all(np.abs(got - want) <= BF * 1.01 * (ref.gated_ff(h[0], h[2], h[3], h[4], None, "relu")[2] + np.abs(want)))
        for n in d:
            assert np.all(np.abs(host(d[n]) - back[n]) <= BF * 1.01 * (back[n + "_stored"] + np.abs(back[n]))), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,F,H,Fo", [(100, 16, 24, 40), (77, 31, 40, 99), (5000, 128, 300, 128)])
def test_dropout_behind_the_block(single, dtype, rows, F, H, Fo):
    """The block's mask is the one of gnnco_dropout; kept results are scaled, dropped gradients do not come back."""
    t = make(rows, 1, F, H, Fo, dtype)
    drop = gnnco.Dropout(0.25, 77, layer=4, step=9)
    mask = ref.keep(rows, Fo, 0.25, 77, 4, 9) / 0.75
    y = check_forward(single, t, None, "silu", dtype, drop, mask)
    assert np.array_equal(host(y) != 0, mask != 0)
    check_backward(single, t, None, "silu", dtype, drop, mask, slots=16)
    nothing = gnnco.Dropout(1.0, 77)
    assert not single.gated_ff(t[0], *t[2:], drop=nothing).any()
    d = single.gated_ff_backward(*t, drop=nothing)
    assert not any(v.any() for v in d.values())


@pytest.mark.parametrize("rows", [60, 6000])
def test_float32_weights_of_bfloat16_features(single, rows):
    import torch
    t = make(rows, 1, 72, 200, 40, "bf16", w_dtype="f32")
    check_forward(single, t, None, "gelu", "bf16")
    d = check_backward(single, t, None, "gelu", "bf16", slots=16)
    assert d["dw_up"].dtype == torch.float32 and d["dx"].dtype == torch.bfloat16
    e = check_backward(single, t, None, "gelu", "bf16", slots=16, dw_dtype=torch.bfloat16)
    assert torch.equal(e["dw_up"], d["dw_up"].bfloat16())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,offset", [(48, 0), (48, 8), (41, 0), (41, 1), (42, 2), (44, 4)])
def test_columns_of_wider_tensors(single, dtype, ld, offset):
    import torch
    rows, F, H = 150, 40, 56
    t = make(rows, 1, F, H, F, dtype)
    want, want_d = single.gated_ff(t[0], *t[2:]), single.gated_ff_backward(*t)
    wide = [torch.full((rows, ld + offset), 7.0, dtype=t[0].dtype, device="cuda") for _ in range(4)]
    x, dy, y, dx = (w[:, offset:offset + F] for w in wide)
    x.copy_(t[0])
    dy.copy_(t[1])
    single.gated_ff(x, *t[2:], out=y)
    d = single.gated_ff_backward(x, dy, *t[2:], dx=dx)
    assert torch.equal(y, want) and torch.equal(dx, want_d["dx"])
    for n in ("dw_gate", "dw_up", "dw_down"):
        assert torch.equal(d[n], want_d[n])
    for w in wide:
        w[:, offset:offset + F] = 7.0
        assert bool((w == 7.0).all())


def test_unaligned_weights(single):
    import torch
    t = make(70, 1, 40, 56, 40, "bf16")
    want = single.gated_ff(t[0], *t[2:])
    moved = []
    for w in t[2:]:
        flat = torch.empty(w.numel() + 1, dtype=w.dtype, device="cuda")
        flat[1:] = w.flatten()
        moved.append(flat[1:].view(w.shape))
    assert torch.equal(single.gated_ff(t[0], *moved), want)


def test_in_place_and_partial_wishes(single):
    import torch
    for dtype in ("f32", "bf16"):
        t = make(600, 1, 64, 96, 64, dtype)
        want, d = single.gated_ff(t[0], *t[2:]), single.gated_ff_backward(*t)
        for aliased in (0, 1):
            u = [v.clone() for v in t]
            e = single.gated_ff_backward(*u, dx=u[aliased])
            assert all(torch.equal(e[k], d[k]) for k in d)
        assert torch.equal(single.gated_ff_backward(*t, want_dw=False)["dx"], d["dx"])
        assert torch.equal(single.gated_ff_backward(*t, want_dx=False)["dw_down"], d["dw_down"])
        x = t[0].clone()
        single.gated_ff(x, *t[2:], out=x)
        assert torch.equal(x, want)


def test_no_rows(single):
    t = make(0, 1, 16, 24, 8, "f32")
    assert single.gated_ff(t[0], *t[2:]).shape == (0, 8)
    d = single.gated_ff_backward(*t)
    assert d["dx"].shape == (0, 16) and not d["dw_gate"].any() and not d["dw_down"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nans_stay_in_their_rows_and_sets(dtype):
    import torch
    sizes = [70, 1, 130, 5]
    ptr = np.concatenate([[0], np.cumsum(sizes)])
    g = load(sizes)
    t = make(206, 4, 24, 40, 16, dtype)
    want, d = g.gated_ff(t[0], *t[2:]), g.gated_ff_backward(*t)
    x = t[0].clone()
    x[75, 3], x[71, 0] = float("nan"), float("inf")            # rows of set 2
    y, e = g.gated_ff(x, *t[2:]), g.gated_ff_backward(x, *t[1:])
    rest = torch.ones(206, dtype=torch.bool)
    rest[[71, 75]] = False
    assert torch.equal(y[rest.cuda()], want[rest.cuda()]) and torch.equal(e["dx"][rest.cuda()], d["dx"][rest.cuda()])
    assert bool(torch.isnan(y[75]).all())
    for n in ("dw_gate", "dw_up", "dw_down"):
        assert all(torch.equal(e[n][s], d[n][s]) for s in (0, 1, 3)) and bool(torch.isnan(e[n][2]).any())
    w = [v.clone() for v in t[2:]]
    w[0][1].fill_(float("nan"))                                # a set's weights spoil its own rows only
    y = g.gated_ff(t[0], *w)
    assert bool(torch.isnan(y[70]).all())
    others = torch.cat([y[:70], y[71:]])
    assert torch.equal(others, torch.cat([want[:70], want[71:]]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_runs_agree_bit_by_bit_and_on_other_streams(dtype):
    import torch
    sizes = [3000, 40, 0, 2777]
    g = load(sizes)
    t = make(sum(sizes), 4, 72, 136, 72, dtype)
    want, d = g.gated_ff(t[0], *t[2:]), g.gated_ff_backward(*t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, e = g.gated_ff(t[0], *t[2:], stream=side), g.gated_ff_backward(*t, stream=side)
    side.synchronize()
    assert torch.equal(y, want) and all(torch.equal(d[k], e[k]) for k in d)


def test_work_areas(single):
    import torch
    t = make(50, 1, 16, 24, 8, "f32")
    want = single.gated_ff(t[0], *t[2:])
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert torch.equal(single.gated_ff(t[0], *t[2:], ws=ws), want)
    with pytest.raises(gnnco.GnncoError) as e:
        single.gated_ff(t[0], *t[2:], ws=ws[:256])
    assert e.value.status == gnnco.WORKSPACE_TOO_SMALL
    with pytest.raises(gnnco.GnncoError) as e:
        single.gated_ff(t[0], *t[2:], ws=ws[1:])
    assert e.value.status == gnnco.INVALID_ARGUMENT


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_recorded_graphs_replay_with_new_inputs(single, dtype):
    import torch
    t, u = make(700, 1, 64, 96, 64, dtype, 1), make(700, 1, 64, 96, 64, dtype, 2)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    drop = gnnco.Dropout(0.3, 5, step_dev=step)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        single.gated_ff_backward(*t, drop=drop)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        y, d = single.gated_ff(t[0], *t[2:], drop=drop), single.gated_ff_backward(*t, drop=drop)
        step.add_(1)
    for k in range(2):
        if k:
            for a, b in zip(t, u):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        eager = gnnco.Dropout(0.3, 5, step=k)
        assert torch.equal(y, single.gated_ff(t[0], *t[2:], drop=eager))
        e = single.gated_ff_backward(*t, drop=eager)
        assert all(torch.equal(d[n], e[n]) for n in d)


def test_gradients_against_differences(single):
    """float32: the directional derivative of the loss <y, dy> by differences of the library's own forward pass, in x and each weight."""
    import torch
    t = make(64, 1, 24, 40, 16, "f32")
    d = single.gated_ff_backward(*t)

    def loss(x, wg, wu, wd):
        return (single.gated_ff(x, wg, wu, wd).double() * t[1].double()).sum().item()

    base = [t[0], *t[2:]]
    r = torch.Generator(device="cuda").manual_seed(4)
    for i, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down")):
        v = torch.randn(base[i].shape, device="cuda", generator=r)
        e = 2.0 ** -7
        up, low = ([b + s * e * v if j == i else b for j, b in enumerate(base)] for s in (1, -1))
        want = (loss(*up) - loss(*low)) / (2 * e)
        got = (d[name].double() * v.double()).sum().item()
        # the third derivative along v leaves e^2 / 6 of its size (the loss is of order 100), rounding 2^-24 * 100 / e
        assert abs(got - want) <= 0.03 + 0.003 * abs(want), name


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("F,H,Fo", [(1, 1, 1), (40, 56, 24), (1024, 4096, 1024), (99, 343, 51), (2048, 64, 512), (64, 3000, 8), (5000, 33, 16)])
@pytest.mark.parametrize("dtype,w_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_few_rows(single, rows, F, H, Fo, dtype, w_dtype):
    """One to four rows have kernels of their own; a row does not depend on the others."""
    import torch
    t = make(rows, 1, F, H, Fo, dtype, seed=rows, w_dtype=w_dtype)
    act = ("silu", "gelu")[rows % 2]
    y = check_forward(single, t, None, act, dtype)
    drop = gnnco.Dropout(0.4, 3, layer=1)
    mask = ref.keep(rows, Fo, 0.4, 3, 1) / 0.6
    z = check_forward(single, t, None, act, dtype, drop, mask)
    assert np.array_equal(host(z) != 0, (mask != 0) & (host(y) != 0))
    if rows == 4:
        x = t[0].clone()
        x[1] = float("nan")
        assert torch.equal(single.gated_ff(x, *t[2:], act=act)[[0, 2, 3]], y[[0, 2, 3]])
        wide = torch.empty(rows, F + 3, dtype=t[0].dtype, device="cuda")
        wide[:, 1:F + 1] = t[0]
        out = torch.empty(rows, Fo + 5, dtype=t[0].dtype, device="cuda")
        single.gated_ff(wide[:, 1:F + 1], *t[2:], act=act, out=out[:, 2:Fo + 2])
        assert torch.equal(out[:, 2:Fo + 2], y)


@pytest.mark.parametrize("F,H,Fo", [(256, 512, 256), (64, 64, 64), (40, 65, 24), (130, 200, 257), (136, 136, 136), (8, 1, 8), (250, 130, 129), (200, 1000, 72)])
@pytest.mark.parametrize("act,p", [("silu", 0.0), ("gelu", 0.3), ("silu", 0.1)])
def test_many_rows_in_bfloat16(F, H, Fo, act, p):
    """Enough tiles of 256 rows for every pair of CTAs: widths up to 256 run as one kernel, in which several tiles follow each
    other; ragged and empty subgraphs, odd and even numbers of chunks of h."""
    sizes = [300, 0, 257, 1, 33, 5000, 256] * 6 + [640] * 10
    ptr = np.concatenate([[0], np.cumsum(sizes)])
    g = load(sizes)
    rows = int(ptr[-1])
    drop = gnnco.Dropout(p, 21, layer=2, step=3) if p else None
    mask = ref.keep(rows, Fo, p, 21, 2, 3) / (1 - p) if p else None
    t = make(rows, len(sizes), F, H, Fo, "bf16", seed=H)
    y = check_forward(g, t, ptr, act, "bf16", drop, mask)
    if p:
        assert not host(y)[mask == 0].any()
    u = make(rows, 1, F, H, Fo, "bf16", seed=H + 1)
    check_forward(g, u, None, act, "bf16", drop, mask)
    assert g.async_status() == gnnco.OK


def test_in_place_as_one_kernel():
    import torch
    sizes = [300, 257, 40] * 60
    g = load(sizes)
    t = make(sum(sizes), len(sizes), 96, 200, 96, "bf16")
    want = g.gated_ff(t[0], *t[2:])
    x = t[0].clone()
    g.gated_ff(x, *t[2:], out=x)
    assert torch.equal(x, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradients_of_more_rows_than_one_run_takes(single, dtype):
    """150,000 rows with one set: three runs at least, whose sums are joined.  Sums of that many terms are compared with the same
    products in float64 on the GPU, by norm: float32's chains of some thousand roundings are random."""
    import torch
    rows, F, H = 150_001, 72, 40
    t = make(rows, 1, F, H, F, dtype)
    d = single.gated_ff_backward(*t, dw_dtype=torch.float32)
    x, dy, wg, wu, wd = (v.double() for v in t)
    wg, wu, wd = wg[0], wu[0], wd[0]
    g, u, dh = x @ wg, x @ wu, dy @ wd.T
    s = torch.sigmoid(g)
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    want = dict(dx=dg @ wg.T + du @ wu.T, dw_gate=x.T @ dg, dw_up=x.T @ du, dw_down=(g * s * u).T @ dy)
    for n, v in want.items():
        err = float((d[n].double().view_as(v) - v).norm() / v.norm())
        # bfloat16: the stored operand is off by 2^-8 at most, 1.7e-3 in the mean square, and dx once more
        assert err < (2e-6 if dtype == "f32" else 2.6e-3 if n == "dx" else 2e-3), (n, err)


def test_elements_past_32_bits():
    """x, y and the stored h, dg, du have more than 2^31 elements: the last rows against a call on them alone."""
    import torch
    free = torch.cuda.mem_get_info()[0]
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    rows, F, H = (1 << 23) + 4097, 256, 272
    g = load([rows])
    r = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(rows, F, dtype=torch.bfloat16, device="cuda").normal_(generator=r)
    w = [torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=r).mul_(1 / 16) for s in ((1, F, H), (1, F, H), (1, H, F))]
    last = x[-300:].clone()
    drop = gnnco.Dropout(0.5, 11)
    keep = torch.from_numpy(ref.keep(300, F, 0.5, 11, row0=rows - 300)).cuda()
    y = g.gated_ff(x, *w, drop=drop)
    want = torch.where(keep, g.gated_ff(last, *w).float() * 2.0, 0.0)
    assert float((y[-300:].float() - want).norm() / want.norm()) < 2 * BF
    assert torch.equal(y[-300:] != 0, (want != 0) & keep)
    del y
    dx = g.gated_ff_backward(x, x, *w, want_dw=False)["dx"]
    want = g.gated_ff_backward(last, last, *w, want_dw=False)["dx"]
    assert float((dx[-300:].float() - want.float()).norm() / want.float().norm()) < 2 * BF
    assert g.async_status() == gnnco.OK


@pytest.mark.parametrize("F,H,Fo", [(128, 256, 128), (64, 64, 64), (8, 1, 8), (40, 65, 104), (99, 130, 65), (128, 250, 24), (24, 200, 128)])
@pytest.mark.parametrize("act,p", [("silu", 0.0), ("gelu", 0.3)])
def test_gradients_of_many_rows_in_bfloat16(F, H, Fo, act, p):
    """More tiles of rows than SMs, ragged and empty subgraphs; dx in a wider tensor, beside columns that keep their values; dx in
    the place of x, where it may not be written before the weights' gradients have read x, gives the same bits."""
    import torch
    sizes = np.random.RandomState(F + H).randint(0, 1500, 40)
    sizes[[3, 17]] = 0, 1
    ptr = np.concatenate([[0], np.cumsum(sizes)])
    rows = int(ptr[-1])
    g, t = load(sizes), make(rows, len(sizes), F, H, Fo, "bf16")
    drop = gnnco.Dropout(p, 5, layer=2) if p else None
    mask = ref.keep(rows, Fo, p, 5, layer=2) / (1 - p) if p else None
    d = check_backward(g, t, ptr, act, "bf16", drop, mask, slots=4)
    wide = torch.full((rows, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    e = g.gated_ff_backward(*t, act=act, drop=drop, dx=wide[:, :F])
    assert all(torch.equal(e[k], d[k]) for k in d) and bool((wide[:, F:] == 7.0).all())
    e = g.gated_ff_backward(*t, act=act, drop=drop, want_dw=False, dx=wide[:, 1:F + 1])
    assert torch.equal(e["dx"], d["dx"])
    e = g.gated_ff_backward(*t, act=act, drop=drop, dx=t[0])
    assert all(torch.equal(e[k], d[k]) for k in d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,F,H,Fo", [(150, 99, 41, 51), (7000, 99, 200, 51), (7000, 30, 300, 201), (7000, 261, 40, 270)])
def test_odd_columns_of_wider_tensors(single, dtype, rows, F, H, Fo):
    """Rows start on 16 bytes but end inside 16: what lies behind them is neither read (it is NaN) nor written."""
    import torch
    x, dy, *w = make(rows, 1, F, H, Fo, dtype)

    def wide(t):
        full = torch.full((rows, 272), float("nan"), dtype=t.dtype, device="cuda")
        full[:, :t.shape[1]] = t
        return full, full[:, :t.shape[1]]
    want, d = single.gated_ff(x, *w), single.gated_ff_backward(x, dy, *w)
    fx, vx = wide(x)
    fdy, vdy = wide(dy)
    fy, vy = wide(torch.zeros_like(dy))
    fdx, vdx = wide(torch.zeros_like(x))
    single.gated_ff(vx, *w, out=vy)
    e = single.gated_ff_backward(vx, vdy, *w, dx=vdx)
    assert torch.equal(vy, want) and all(torch.equal(e[k], d[k]) for k in d)
    for full, n in ((fx, F), (fdy, Fo), (fy, Fo), (fdx, F)):
        assert bool(full[:, n:].isnan().all())


FEW = [0, 1, 8, 9, 2, 16, 17, 3, 0, 7, 60] + [1] * 12


@pytest.mark.parametrize("F,H,Fo", [(1, 1, 1), (33, 19, 21), (64, 128, 40), (384, 40, 100), (20, 1024, 384), (32, 65, 33)])
@pytest.mark.parametrize("act,p", [("silu", 0.0), ("gelu", 0.3)])
def test_subgraphs_of_few_rows_in_float32(F, H, Fo, act, p):
    """Sums of eight partial sums, K / 8 roundings each, are inside the bound of the tiled products for these lengths (18 + K / 64 on g
    and u, three times over in the backward pass, from K = 384: 56)."""
    import torch
    ptr = np.concatenate([[0], np.cumsum(FEW)])
    rows = int(ptr[-1])
    g, t = load(FEW), make(rows, len(FEW), F, H, Fo, "f32")
    drop = gnnco.Dropout(p, 5, layer=2) if p else None
    mask = ref.keep(rows, Fo, p, 5, layer=2) / (1 - p) if p else None
    y = check_forward(g, t, ptr, act, "f32", drop, mask)
    d = check_backward(g, t, ptr, act, "f32", drop, mask, slots=8)
    assert all(not d[k][s].any() for k in ("dw_gate", "dw_up", "dw_down") for s in (0, 8))
    wide = torch.full((rows, 401), 7.0, device="cuda")
    x = wide[:, 1:F + 1]
    x.copy_(t[0])
    assert torch.equal(g.gated_ff(x, *t[2:], act=act, drop=drop), y)
    e = g.gated_ff_backward(x, t[1], *t[2:], act=act, drop=drop, dx=x)
    assert all(torch.equal(e[k], d[k]) for k in d)
    assert bool((wide[:, F + 1:] == 7.0).all()) and bool((wide[:, 0] == 7.0).all())
    assert torch.equal(g.gated_ff_backward(*t, act=act, drop=drop, want_dw=False)["dx"], d["dx"])
    assert torch.equal(g.gated_ff_backward(*t, act=act, drop=drop, want_dx=False)["dw_up"], d["dw_up"])
    check_backward(g, t, ptr, act, "f32", drop, mask, slots=8, dw_dtype=torch.bfloat16)
    bad = [v.clone() for v in t]
    bad[0][int(ptr[3])] = float("nan")                      # a row of subgraph 3
    bad[2][1] = float("inf")                                # the gate's weights of subgraph 1
    y2, d2 = g.gated_ff(bad[0], *bad[2:], act=act), g.gated_ff_backward(*bad, act=act)
    y, d = g.gated_ff(t[0], *t[2:], act=act), g.gated_ff_backward(*t, act=act)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[int(ptr[3])] = keep[int(ptr[1])] = False
    assert torch.equal(y2[keep], y[keep]) and torch.equal(d2["dx"][keep], d["dx"][keep])
    sets = [s for s in range(len(FEW)) if s not in (1, 3)]
    assert all(torch.equal(d2[k][sets], d[k][sets]) for k in ("dw_gate", "dw_up", "dw_down"))
