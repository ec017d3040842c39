"""Plain float64 restatements (numpy) of dropout and of the gated feed-forward block; they share no code with the library."""
import math

import numpy as np


def philox(counter, key, rounds=10):
    """Philox4x32 of counters [n, 4] under the key (two words): [n, 4], all numpy uint64 below 2^32."""
    c = [counter[:, i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=1)


def keep(rows, F, p, seed, layer=0, step=0, row0=0):
    """Which elements of rows row0 .. row0 + rows stay."""
    quads = -(-F // 4)
    n = np.arange(rows * quads, dtype=np.uint64) + np.uint64(row0 * quads)
    counter = np.stack([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), np.full_like(n, step), np.full_like(n, layer)], axis=1)
    words = philox(counter, (seed & 0xFFFFFFFF, seed >> 32)).reshape(rows, quads * 4)[:, :F]
    return words >= np.uint64(round(p * 2.0 ** 32))


def dropout(x, p, seed, layer=0, step=0):
    on = keep(x.shape[0], x.shape[1], p, seed, layer, step)
    return np.where(on, x.astype(np.float64) * (1.0 / (1.0 - p) if p < 1.0 else 0.0), 0.0)


def _erf(v):
    import torch
    return torch.erf(torch.from_numpy(np.ascontiguousarray(v, dtype=np.float64))).numpy()


def act(name, g):
    """The activation and its derivative."""
    if name == "relu":
        return np.maximum(g, 0.0), (g > 0.0).astype(np.float64)
    if name == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    phi = 0.5 * (1.0 + _erf(g / math.sqrt(2.0)))
    return g * phi, phi + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def ranges(part_ptr, sets, rows):
    return [(0, rows)] if sets == 1 else [(int(part_ptr[s]), int(part_ptr[s + 1])) for s in range(sets)]


def gated_ff(x, wg, wu, wd, ptr, name, mask=None):
    """(y, mag, stored): x [rows, F], weights [sets, ..], ptr [sets + 1] first row of every set (sets > 1), mask
    [rows, F_out]: 0 or 1 / (1 - p).  mag: sum of the sizes of y's terms, cancellation inside g and u undone;
    stored: what an error of h relative to itself makes of y."""
    x, wg, wu, wd = (t.astype(np.float64) for t in (x, wg, wu, wd))
    y = np.zeros((x.shape[0], wd.shape[2]))
    mag, stored = np.zeros_like(y), np.zeros_like(y)
    for s, (a, b) in enumerate(ranges(ptr, wg.shape[0], x.shape[0])):
        g, u = x[a:b] @ wg[s], x[a:b] @ wu[s]
        h = act(name, g)[0] * u
        y[a:b] = h @ wd[s]
        gm, um = np.abs(x[a:b]) @ np.abs(wg[s]), np.abs(x[a:b]) @ np.abs(wu[s])
        mag[a:b] = (gm * um) @ np.abs(wd[s])
        stored[a:b] = np.abs(h) @ np.abs(wd[s])
    return (y, mag, stored) if mask is None else (y * mask, mag * mask, stored * mask)


def gated_ff_backward(x, dy, wg, wu, wd, ptr, name, mask=None):
    """dict of the gradients, and under name + '_mag' and name + '_stored' the same sizes for them (errors of h, dg, du)."""
    x, dy, wg, wu, wd = (t.astype(np.float64) for t in (x, dy, wg, wu, wd))
    if mask is not None:
        dy = dy * mask
    out = dict(dx=np.zeros_like(x), dw_gate=np.zeros_like(wg), dw_up=np.zeros_like(wu), dw_down=np.zeros_like(wd))
    for k, v in list(out.items()):
        out[k + "_mag"], out[k + "_stored"] = np.zeros_like(v), np.zeros_like(v)
    for s, (a, b) in enumerate(ranges(ptr, wg.shape[0], x.shape[0])):
        xs, ds = x[a:b], dy[a:b]
        g, u, dh = xs @ wg[s], xs @ wu[s], ds @ wd[s].T
        f, slope = act(name, g)
        dg, du, h = dh * u * slope, dh * f, f * u
        out["dx"][a:b] = dg @ wg[s].T + du @ wu[s].T
        out["dw_gate"][s], out["dw_up"][s], out["dw_down"][s] = xs.T @ dg, xs.T @ du, h.T @ ds
        xm, dm, gw, uw, dw = (np.abs(t) for t in (xs, ds, wg[s], wu[s], wd[s]))
        out["dx_stored"][a:b] = np.abs(dg) @ gw.T + np.abs(du) @ uw.T
        out["dw_gate_stored"][s], out["dw_up_stored"][s], out["dw_down_stored"][s] = xm.T @ np.abs(dg), xm.T @ np.abs(du), np.abs(h).T @ dm
        gm, um, hm = xm @ gw, xm @ uw, dm @ dw.T
        # |act'| and |act''| are below 1.2 (1.13 and 0.8 at most): a change of g by e changes dg by less than 1.2 |dh u| e
        dgm, dum = 1.2 * hm * um * (1.0 + gm), 1.2 * hm * gm
        out["dx_mag"][a:b] = dgm @ gw.T + dum @ uw.T
        out["dw_gate_mag"][s], out["dw_up_mag"][s], out["dw_down_mag"][s] = xm.T @ dgm, xm.T @ dum, (1.2 * gm * um).T @ dm
    return out
