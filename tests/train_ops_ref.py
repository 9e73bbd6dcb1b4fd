"""64-bit definitions of the operators beside the step (not a test module): token log-probabilities, the residual junction
and the orthogonalised update, written from their formulas with numpy."""
import numpy as np

NS = (3.4445, -4.7750, 2.0315)
U32 = 2.0 ** -24
U16 = 2.0 ** -11        # half a step of fp16, relative


def token_logprobs(x, tok, temp, n_top):
    """x [rows, vocab] fp64; returns logp, entropy, (max, L), ids, top values, row by row."""
    rows, vocab = x.shape
    logp, ent, stats = np.zeros(rows), np.zeros(rows), np.zeros((2, rows))
    ids, vals = np.full((rows, n_top), -1, np.int64), np.full((rows, n_top), -np.inf)
    for r in range(rows):
        t, z = tok[r], x[r]
        if t < 0 or t >= vocab:
            continue
        if np.isnan(z).any() or np.isposinf(z).any():
            logp[r] = ent[r] = stats[0, r] = stats[1, r] = np.nan
            vals[r] = np.nan
            continue
        m = z.max()
        if np.isneginf(m):
            logp[r], stats[0, r] = -np.inf, -np.inf
            continue
        e = (z - m) / temp
        rest = np.exp(np.delete(e, int(np.argmax(z)))).sum()
        L = np.log1p(rest)
        q = e - L
        p = np.exp(q)
        logp[r], stats[0, r], stats[1, r] = q[t], m, L
        ent[r] = -(p[p > 0] * q[p > 0]).sum()
        order = np.lexsort((np.arange(vocab), -z))[:n_top]
        order = order[~np.isneginf(z[order])]
        ids[r, :len(order)], vals[r, :len(order)] = order, q[order]
    return logp, ent, stats, ids, vals


def token_logprobs_bwd(x, tok, temp, stats, ent, g, h, ld):
    """The gradient from given statistics (max, L) and entropy; [rows, ld]."""
    rows, vocab = x.shape
    out = np.zeros((rows, ld))
    for r in range(rows):
        if tok[r] < 0 or tok[r] >= vocab or np.isneginf(stats[0, r]):
            continue
        q = (x[r] - stats[0, r]) / temp - stats[1, r]
        p = np.exp(q)
        d = -p * g[r]
        d[tok[r]] = -np.expm1(q[tok[r]]) * g[r]
        live = p > 0
        d[live] -= h[r] * p[live] * (q[live] + ent[r])
        out[r, :vocab] = d / temp
    return out


def norm(t, kind, eps, gain, bias):
    mean = t.mean(1) if kind == 0 else np.zeros(len(t))
    rstd = 1.0 / np.sqrt(((t - mean[:, None]) ** 2).mean(1) + eps)
    hat = (t - mean[:, None]) * rstd[:, None]
    return hat * gain + (bias if kind == 0 else 0.0), hat, mean, rstd


def join_fwd(kind, eps, scale, x, h, gain1, bias1, gate, rpg, gain2, bias2):
    """Returns x', y, stats [4, rows], and what the gradient's tolerances need (hat1, hat2, u, gate rows)."""
    rows = len(x)
    st = np.zeros((4, rows))
    u, hat1 = h, None
    if gain1 is not None:
        u, hat1, st[0], st[1] = norm(h, kind, eps, gain1, bias1)
    q = np.ones_like(h) if gate is None else gate[np.arange(rows) // rpg]
    xo = scale * x + q * u
    y = hat2 = None
    if gain2 is not None:
        y, hat2, st[2], st[3] = norm(xo, kind, eps, gain2, bias2)
    return xo, y, st, (hat1, hat2, u, q)


def norm_bwd(v, hat, rstd, gain, kind):
    w = v * gain
    d = w - hat * (w * hat).mean(1, keepdims=True)
    if kind == 0:
        d = d - w.mean(1, keepdims=True)
    return d * rstd[:, None]


def join_bwd(kind, scale, dy, dxo, xo, h, st, gain1, bias1, gate, rpg, gain2):
    """From the statistics the forward pass saved.  Returns a dict of the gradients."""
    rows, out = len(h), {}
    d = np.zeros_like(h) if dxo is None else dxo.copy()
    if gain2 is not None:
        hat2 = (xo - st[2][:, None]) * st[3][:, None]
        out["dgain2"], out["dbias2"] = (dy * hat2).sum(0), dy.sum(0)
        d += norm_bwd(dy, hat2, st[3], gain2, kind)
    out["dx"], out["d"] = scale * d, d
    u = h
    if gain1 is not None:
        hat1 = (h - st[0][:, None]) * st[1][:, None]
        u = hat1 * gain1 + (bias1 if kind == 0 else 0.0)
    du = d
    if gate is not None:
        out["dgate"] = np.stack([(d * u)[i:i + rpg].sum(0) for i in range(0, rows, rpg)])
        du = d * gate[np.arange(rows) // rpg]
    out["du"] = du
    if gain1 is not None:
        out["dgain1"], out["dbias1"] = (du * hat1).sum(0), du.sum(0)
        du = norm_bwd(du, hat1, st[1], gain1, kind)
    out["dh"] = du
    return out


def orthogonalize(g, steps=5):
    a, b, c = NS
    x = g / max(np.linalg.norm(g), 1e-30)
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            A = x @ x.T
            x = a * x + (b * A + c * (A @ A)) @ x
        else:
            A = x.T @ x
            x = a * x + x @ (b * A + c * (A @ A))
    return x


def muon_step(master, grad, mom, lr, mu, nesterov, wd, steps=5):
    mom = mu * mom + grad
    u = grad + mu * mom if nesterov else mom
    return master * (1 - lr * wd) - lr * 0.2 * np.sqrt(max(master.shape)) * orthogonalize(u, steps), mom
