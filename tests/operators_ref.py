"""Plain float64 restatements (numpy) of the embedding, block-norm and orthogonalised-update operators; they share no
code with the library."""
import numpy as np


def lookup(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t].astype(np.float64)
    return out


def table_grad(dout, tokens, V, scale):
    """(gradient, sum of magnitudes, rows per token): the second and third give the rounding bound of the sum."""
    g, mag, cnt = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V)
    for i, t in enumerate(tokens):
        if 0 <= t < V:
            g[t] += dout[i].astype(np.float64)
            mag[t] += np.abs(dout[i].astype(np.float64))
            cnt[t] += 1
    return scale * g, abs(scale) * mag, cnt


def _r(v, eps):
    return 1.0 / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)


def block_norm(x, y, gate, w_pre, w_post, scale, eps):
    x = x.astype(np.float64)
    if y is not None:
        y = y.astype(np.float64)
        x = x + scale * (1.0 if gate is None else gate.astype(np.float64)) * (y * _r(y, eps)) * (1.0 if w_post is None else w_post)
    return x, x * _r(x, eps) * (1.0 if w_pre is None else w_pre)


def block_norm_backward(x, y, gate, w_pre, w_post, scale, eps, dx_out, dh):
    """x: the stream after the block.  Returns the gradients and, under the same names + '_mag', for the sums over rows
    the sums of the terms' magnitudes."""
    x = x.astype(np.float64)
    w1 = 1.0 if w_pre is None else w_pre.astype(np.float64)
    r = _r(x, eps)
    xh = x * r
    dh = np.zeros_like(x) if dh is None else dh.astype(np.float64)
    a = dh * w1
    D = r * (a - xh * (a * xh).mean(axis=1, keepdims=True))
    if dx_out is not None:
        D = D + dx_out.astype(np.float64)
    out = dict(dx=D, dw_pre=(dh * xh).sum(0), dw_pre_mag=np.abs(dh * xh).sum(0))
    if y is not None:
        y = y.astype(np.float64)
        g = 1.0 if gate is None else gate.astype(np.float64)
        w2 = 1.0 if w_post is None else w_post.astype(np.float64)
        ry = _r(y, eps)
        yh = y * ry
        b = scale * g * w2 * D
        out["dy"] = ry * (b - yh * (b * yh).mean(axis=1, keepdims=True))
        out["dw_post"], out["dw_post_mag"] = (scale * g * D * yh).sum(0), np.abs(scale * g * D * yh).sum(0)
        dg = scale * w2 * D * yh
        if gate is not None:
            out["dgate"] = dg.sum(0) if gate.ndim == 1 else dg
            out["dgate_mag"] = np.abs(dg).sum(0)
    return out


def newton_schulz(G, steps, coefs, eps):
    """G [sets, r, c] -> the iterate, the definition step by step."""
    G = G.astype(np.float64)
    out = np.empty_like(G)
    for s in range(G.shape[0]):
        X = G[s].T if G.shape[1] > G.shape[2] else G[s]
        X = X / (np.sqrt((X * X).sum()) + eps)
        for _ in range(steps):
            A = X @ X.T
            X = coefs[0] * X + (coefs[1] * A + coefs[2] * (A @ A)) @ X
        out[s] = X.T if G.shape[1] > G.shape[2] else X
    return out


def muon(W, m, g, lr, momentum, nesterov, decay, steps, coefs, eps):
    m = momentum * m.astype(np.float64) + g
    u = g + momentum * m if nesterov else m
    r, c = W.shape[1:]
    o = newton_schulz(u, steps, coefs, eps)
    return W.astype(np.float64) * (1.0 - lr * decay) - lr * np.sqrt(max(1.0, c / r)) * o, m
