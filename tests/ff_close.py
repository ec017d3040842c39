"""How far results of the gated feed-forward block may be off where errors of single terms are independent: sums of n terms are
compared in units of the root of the sum of the terms' squares, not of the sum of their sizes, which grows past the results themselves
when products are chained.  Numpy only; shares no code with the library.

A result carries (stored) errors of the stored h, dg, du, one rounding each, and (inner) errors of the float32 sums and activations
before them.  ``stored`` and ``inner`` below are what relative errors of size 1 of independent signs make of the result.
"""
import numpy as np

import ff_ref as ref

U = 2.0 ** -24
BF = 2.0 ** -8                # half a step of bfloat16, relative
# Independent errors e_k, |e_k| <= c_k, of either sign: |sum e_k| > t sqrt(sum c_k^2) with a probability of at most 2 exp(-t^2 / 2)
# (Hoeffding), 1e-15 at 8.4: below 1e-6 for 10^9 elements.
ELEMENT = 8.4


def _sq(*pairs):
    """sqrt(sum of a^2 b^2) for matrix products a b."""
    return np.sqrt(sum((a * a) @ (b * b) for a, b in pairs))


def _inner(x, wg, wu, name):
    g, u = x @ wg, x @ wu
    a, slope = ref.act(name, g)
    eg, eu = _sq((x, wg)), _sq((x, wu))
    return g, u, a, slope, eg, eu


def forward(x, wg, wu, wd, ptr, name, mask=None):
    """(y, stored, inner), all [rows, F_out]."""
    x, wg, wu, wd = (t.astype(np.float64) for t in (x, wg, wu, wd))
    out = [np.zeros((x.shape[0], wd.shape[2])) for _ in range(3)]
    for s, (lo, hi) in enumerate(ref.ranges(ptr, wg.shape[0], x.shape[0])):
        _, u, a, slope, eg, eu = _inner(x[lo:hi], wg[s], wu[s], name)
        h = a * u
        out[0][lo:hi], out[1][lo:hi] = h @ wd[s], _sq((h, wd[s]))
        out[2][lo:hi] = _sq((np.sqrt((slope * u * eg) ** 2 + (a * eu) ** 2 + h * h), wd[s]))
    return tuple(out) if mask is None else tuple(t * mask for t in out)


def backward(x, dy, wg, wu, wd, ptr, name, mask=None):
    """dict of (gradient, stored, inner)."""
    x, dy, wg, wu, wd = (t.astype(np.float64) for t in (x, dy, wg, wu, wd))
    if mask is not None:
        dy = dy * mask
    out = {n: [np.zeros_like(t) for _ in range(3)] for n, t in (("dx", x), ("dw_gate", wg), ("dw_up", wu), ("dw_down", wd))}
    for s, (lo, hi) in enumerate(ref.ranges(ptr, wg.shape[0], x.shape[0])):
        xs, ds = x[lo:hi], dy[lo:hi]
        _, u, a, slope, eg, eu = _inner(xs, wg[s], wu[s], name)
        dh, edh = ds @ wd[s].T, _sq((ds, wd[s].T))
        h, dg, du = a * u, dh * u * slope, dh * a
        # |act''| is below 0.8 (0.5 for SiLU)
        eh = np.sqrt((slope * u * eg) ** 2 + (a * eu) ** 2 + h * h)
        edg = np.sqrt((edh * u * slope) ** 2 + (dh * eu * slope) ** 2 + (0.8 * dh * u * eg) ** 2 + dg * dg)
        edu = np.sqrt((edh * a) ** 2 + (dh * slope * eg) ** 2 + du * du)
        out["dx"][0][lo:hi] = dg @ wg[s].T + du @ wu[s].T
        out["dx"][1][lo:hi] = _sq((dg, wg[s].T), (du, wu[s].T))
        out["dx"][2][lo:hi] = _sq((edg, wg[s].T), (edu, wu[s].T))
        for n, p, v, e, q in (("dw_gate", xs.T, dg, edg, None), ("dw_up", xs.T, du, edu, None), ("dw_down", h.T, ds, eh, ds)):
            out[n][0][s], out[n][1][s] = p @ v, _sq((p, v))
            out[n][2][s] = _sq((p, e)) if q is None else _sq((e.T, q))
    return {n: tuple(v) for n, v in out.items()}


def units(K, dtype):
    """Errors of a sum over K in units of 2^-24 of the root of its terms' squares.  float32 operands: a stage of 64 adds four large products of 16
    terms, cut off twice by at most 2^-23 each, half of that on average (8; plain multiplications of at most K / 8 terms in a row
    stay below that for the tested lengths), and the stages are rounded to nearest when they are added up.  bfloat16 operands: K / 16 additions, cut off twice."""
    return 8 + (K / 64) ** 0.5 if dtype == "f32" else 8 + K / 8


def worst(got, want, dtype, first, last, out_bf16=False, axis=None):
    """The largest part of what is allowed that `got` is off by `want` = (value, stored, inner): element by element, and by norm over all but
    `axis` (the set, for weight gradients).  first, last: lengths of the sums before the stored values and behind them."""
    value, stored, inner = want
    assert got.shape == value.shape and np.all(np.isfinite(got))
    if not got.size:
        return 0.0
    # the activation's fast forms and their derivative, products, masks: 24 roundings at most
    b_in, b_st, b_out = (units(first, dtype) + 24) * U, units(last, dtype) * U, 0.0
    if dtype == "bf16":
        b_st += BF
    if out_bf16:
        b_out = BF
    err = np.abs(got - value)
    bound = ELEMENT * (b_in * inner + b_st * stored) + b_out * np.abs(value) + 1e-35
    ratio = float((err / bound).max())
    over = tuple(i for i in range(value.ndim) if i != axis)
    norm = lambda t: np.sqrt((t * t).sum(axis=over))  # noqa: E731
    bound = b_in * norm(inner) + b_st * norm(stored) + b_out * norm(value) + 1e-35
    return max(ratio, float(np.max(norm(err) / bound)))


def whole_numbers(rows, sets, F, H, Fo, seed=0, ptr=None):
    """x, dy, wg, wu, wd of small integers and so few entries that, with the rectifier and masks scaled by 1 or 2, h (144 at most), dg
    and du (96) are integers of eight bits and every sum over up to 2^24 / 192 rows is one of 24: exact in every type and order."""
    r = np.random.RandomState(seed)
    x, dy = r.randint(-2, 3, (rows, F)), r.randint(-1, 2, (rows, Fo))

    def few(sets, n, cols, per, most):
        """[sets, n, cols]: at most `per` entries in every column"""
        w = np.zeros((sets, n, cols))
        at = r.randint(0, n, (sets, per, cols))
        np.put_along_axis(w, at, r.randint(1, most + 1, at.shape) * r.choice([-1, 1], at.shape), axis=1)
        return w
    return x, dy, few(sets, F, H, 3, 2), few(sets, F, H, 3, 2), np.swapaxes(few(sets, Fo, H, 4, 1), 1, 2)
