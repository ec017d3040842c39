"""What the comparison of ff_close accepts and rejects, on results made on the CPU: arithmetic like the library's passes, wrong results
of the kinds that a kernel with a fault gives do not."""
import numpy as np
import pytest
import torch

import ff_close as close
import ff_ref as ref

F32, BF16 = torch.float32, torch.bfloat16


def draw(rows, F, H, Fo, dtype, seed=0):
    r = np.random.RandomState(seed)
    t = [r.standard_normal(s) * k for s, k in (((rows, F), 1.0), ((rows, Fo), 1.0), ((1, F, H), F ** -0.5), ((1, F, H), F ** -0.5), ((1, H, Fo), H ** -0.5))]
    # (float32 values have more bits than two limbs)
    return [torch.from_numpy(v).to(BF16 if dtype == "bf16" else F32) for v in t]


def np64(t):
    return t.double().numpy()


def act(name, g):
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    phi = 0.5 * torch.erfc(-g / 2 ** 0.5)
    return g * phi, phi + g * torch.exp(-0.5 * g * g) / (2 * np.pi) ** 0.5


def chain(t, name, dtype, slope_of=None, limbs=3):
    """y and the gradients in float32, with the roundings of the library's bfloat16 form; limbs: of every operand of a product."""
    store = (lambda v: v.to(BF16).float()) if dtype == "bf16" else (lambda v: v)

    def cut(v):
        if limbs == 3 or dtype == "bf16":
            return v
        out, rest = torch.zeros_like(v), v
        for _ in range(limbs):
            part = rest.to(BF16).float()
            out, rest = out + part, rest - part
        return out
    x, dy, wg, wu, wd = (cut(v.float()) for v in t)
    wg, wu, wd = wg[0], wu[0], wd[0]
    g, u, dh = x @ wg, x @ wu, dy @ wd.T
    a, slope = act(name, g)
    if slope_of:
        slope = slope_of(g)
    h, dg, du = (cut(store(v)) for v in (a * u, dh * u * slope, dh * a))
    d = dict(y=h @ wd, dx=dg @ wg.T + du @ wu.T, dw_gate=(x.T @ dg)[None], dw_up=(x.T @ du)[None], dw_down=(h.T @ dy)[None])
    return {n: store(v) for n, v in d.items()}


def ratios(got, t, name, dtype, only=None):
    args = [np64(v) for v in t]
    rows, F, H, Fo = args[0].shape[0], args[0].shape[1], args[2].shape[2], args[4].shape[2]
    want = dict(y=close.forward(args[0], *args[2:], None, name), **close.backward(*args, None, name))
    last = dict(y=H, dx=2 * H, dw_gate=rows, dw_up=rows, dw_down=rows)
    return {n: close.worst(np64(got[n]), want[n], dtype, F if n == "y" else max(F, Fo), last[n], dtype == "bf16", 0 if n[:2] == "dw" else None)
            for n in want if only is None or n in only}


SHAPES = [(1, 8, 8, 8), (3, 5, 7, 2), (129, 100, 96, 100), (300, 128, 200, 128), (1000, 99, 343, 99), (65, 24, 1000, 8), (5000, 128, 300, 128)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_right_results_pass(shape, dtype, name):
    t = draw(*shape, dtype)
    r = ratios(chain(t, name, dtype), t, name, dtype)
    assert max(r.values()) <= 1.0, r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5000, 128, 300, 128), (2000, 130, 521, 257), (1500, 264, 640, 200)])
def test_wrong_results_do_not(dtype, shape):
    t = draw(*shape, dtype)
    right = chain(t, "silu", dtype)
    zeros = {n: torch.zeros_like(v) for n, v in right.items()}
    assert min(ratios(zeros, t, "silu", dtype).values()) > 1.0
    # the slope without a (1 - s)
    r = ratios(chain(t, "silu", dtype, slope_of=torch.sigmoid), t, "silu", dtype)
    assert r["dw_gate"] > 1.0 and r["dx"] > 1.0, r
    # a last row that the sums over rows leave out
    short = chain([v[:-1] if i < 2 else v for i, v in enumerate(t)], "silu", dtype)
    r = ratios(short, t, "silu", dtype, ("dw_gate", "dw_up", "dw_down"))
    assert min(r.values()) > 1.0, r
    # a last column of h that is left out
    cut = [v.clone() for v in t]
    cut[4][:, -1] = 0
    r = ratios(chain(cut, "silu", dtype), t, "silu", dtype, ("y", "dx"))
    assert min(r.values()) > 1.0, r
    # a last column and a last row of a result
    for n, v in right.items():
        for index in ((..., -1), (..., -1, slice(None))):
            w = v.clone()
            w[index] = 0
            assert ratios({n: w}, t, "silu", dtype, (n,))[n] > 1.0, (n, index)


@pytest.mark.parametrize("limbs", [1, 2])
def test_float32_results_of_fewer_limbs_do_not_pass(limbs):
    t = draw(1000, 99, 343, 99, "f32")
    r = ratios(chain(t, "gelu", "f32", limbs=limbs), t, "gelu", "f32")
    assert min(r.values()) > 1.0, r


def test_few_rows_of_long_sums():
    t = draw(1, 1024, 4096, 1024, "bf16")
    assert ratios(chain(t, "gelu", "bf16"), t, "gelu", "bf16", ("y",))["y"] <= 1.0
    cut = [v.clone() for v in t]
    cut[4][:, -32:] = 0                                       # the last 32 columns of h
    assert ratios(chain(cut, "gelu", "bf16"), t, "gelu", "bf16", ("y",))["y"] > 1.0


def test_whole_numbers_are_exact_in_bfloat16():
    ptr = [0, 400, 400, 1000]
    x, dy, *w = close.whole_numbers(1000, 3, 20, 70, 33)
    mask = ref.keep(1000, 33, 0.5, 3) * 2.0
    for s, (a, b) in enumerate(zip(ptr, ptr[1:])):
        g, u, dh = x[a:b] @ w[0][s], x[a:b] @ w[1][s], (dy * mask)[a:b] @ w[2][s].T
        for v, most in ((np.maximum(g, 0) * u, 144), (dh * u * (g > 0), 96), (dh * np.maximum(g, 0), 96)):
            assert np.array_equal(v, np.round(v)) and (v.size == 0 or np.abs(v).max() <= most)
    d = ref.gated_ff_backward(x, dy, *w, ptr, "relu", mask)
    assert d["dw_gate"][0].any() and d["dw_down"][2].any() and not d["dw_up"][1].any() and d["dx"].any()
