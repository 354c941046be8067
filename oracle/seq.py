"""TEST INFRASTRUCTURE ONLY: the sequence operators (group norm with an activation, short causal
convolution, selective state space scan, linear attention, gated projection) and their gradients in numpy, 64 bits, written from the
formulas in include/ucd_seq.h and include/ucd_mix.h token by token.  Shares no code with the library.
"""
import numpy as np


def sigmoid(v):
    return np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))


def act_fwd(v, silu):
    return v * sigmoid(v) if silu else v


def act_bwd(v, silu):
    s = sigmoid(v)
    return s * (1 + v * (1 - s)) if silu else np.ones_like(v)


# ---- group norm ------------------------------------------------------------------------------


def norm_fwd(x, gamma, beta, G, eps, silu):
    """(y, mean (N, G), rstd (N, G)) of x (N, S, C)."""
    x = x.astype(np.float64)
    n, s, c = x.shape
    y, mean, rstd = np.empty_like(x), np.empty((n, G)), np.empty((n, G))
    w = c // G
    for i in range(n):
        for g in range(G):
            part = slice(g * w, (g + 1) * w)
            v = x[i, :, part]
            mean[i, g] = v.mean()
            rstd[i, g] = 1 / np.sqrt(((v - mean[i, g]) ** 2).mean() + eps)
            y[i, :, part] = act_fwd(gamma[part] * (v - mean[i, g]) * rstd[i, g] + beta[part], silu)
    return y, mean, rstd


def norm_bwd(x, gamma, beta, G, eps, silu, dy):
    """(dx, dgamma, dbeta)."""
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    _, mean, rstd = norm_fwd(x, gamma, beta, G, eps, silu)
    n, _, c = x.shape
    w = c // G
    dx, dgamma, dbeta = np.empty_like(x), np.zeros(c), np.zeros(c)
    for i in range(n):
        for g in range(G):
            part = slice(g * w, (g + 1) * w)
            xhat = (x[i, :, part] - mean[i, g]) * rstd[i, g]
            du = dy[i, :, part] * act_bwd(gamma[part] * xhat + beta[part], silu)
            dgamma[part] += (du * xhat).sum(0)
            dbeta[part] += du.sum(0)
            dxhat = du * gamma[part]
            dx[i, :, part] = rstd[i, g] * (dxhat - dxhat.mean() - xhat * (dxhat * xhat).mean())
    return dx, dgamma, dbeta


# ---- causal convolution ----------------------------------------------------------------------


def _tokens(x, state, b, n, K):
    """A sequence's tokens behind the K - 1 before it."""
    before = np.zeros((K - 1, x.shape[2])) if state is None else state[b].astype(np.float64)
    return np.concatenate([before, x[b, :n].astype(np.float64)])


def conv_fwd(x, w, bias, silu, lengths=None, state=None):
    """(y, new state): x (B, L, D), w (D, K), state (B, K-1, D)."""
    B, L, D = x.shape
    K = w.shape[1]
    w = w.astype(np.float64)
    bias = np.zeros(D) if bias is None else bias.astype(np.float64)
    y, out = np.zeros((B, L, D)), np.zeros((B, K - 1, D))
    for b in range(B):
        n = L if lengths is None else int(lengths[b])
        xs = _tokens(x, state, b, n, K)
        for t in range(n):
            y[b, t] = act_fwd(bias + sum(w[:, k] * xs[t + k] for k in range(K)), silu)
        out[b] = xs[n:]
    return y, out


def conv_bwd(x, w, bias, silu, dy, lengths=None, state=None, dstate_out=None):
    """(dx, dw, dbias, dstate_in)."""
    B, L, D = x.shape
    K = w.shape[1]
    w = w.astype(np.float64)
    zero = np.zeros(D) if bias is None else bias.astype(np.float64)
    dx, dw, dbias, dstate = np.zeros((B, L, D)), np.zeros((D, K)), np.zeros(D), np.zeros((B, K - 1, D))
    for b in range(B):
        n = L if lengths is None else int(lengths[b])
        xs = _tokens(x, state, b, n, K)
        dxs = np.zeros_like(xs)
        if dstate_out is not None:
            dxs[n:] += dstate_out[b]
        for t in range(n):
            u = zero + sum(w[:, k] * xs[t + k] for k in range(K))
            du = dy[b, t].astype(np.float64) * act_bwd(u, silu)
            dbias += du
            for k in range(K):
                dw[:, k] += du * xs[t + k]
                dxs[t + k] += du * w[:, k]
        dstate[b], dx[b, :n] = dxs[:K - 1], dxs[K - 1:]
    return dx, dw, dbias, dstate


# ---- selective scan --------------------------------------------------------------------------


def _delta(dt, dt_bias, softplus):
    raw = dt.astype(np.float64) + (0 if dt_bias is None else dt_bias.astype(np.float64))
    return (np.logaddexp(0, raw) if softplus else raw), raw


def scan_fwd(u, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, softplus=True, lengths=None, state=None, keep=False):
    """(y, new state): u (B, L, D), A (D, N), Bm (B, L, G, N), state (B, D, N).  keep: also every token's state."""
    B, L, D = u.shape
    N, G = A.shape[1], Bm.shape[2]
    y, out = np.zeros((B, L, D)), np.zeros((B, D, N))
    all_h = np.zeros((B, L + 1, D, N))
    for b in range(B):
        n = L if lengths is None else int(lengths[b])
        h = np.zeros((D, N)) if state is None else state[b].astype(np.float64)
        all_h[b, 0] = h
        for t in range(n):
            ut = u[b, t].astype(np.float64)
            delta, _ = _delta(dt[b, t], dt_bias, softplus)
            bt, ct = (np.repeat(m[b, t].astype(np.float64), D // G, axis=0) for m in (Bm, Cm))
            h = np.exp(delta[:, None] * A) * h + (delta * ut)[:, None] * bt
            all_h[b, t + 1] = h
            y[b, t] = (h * ct).sum(1) + (0 if skip is None else skip * ut)
            if z is not None:
                y[b, t] *= act_fwd(z[b, t].astype(np.float64), True)
        out[b] = h
    return (y, out, all_h) if keep else (y, out)


def scan_bwd(u, dt, A, Bm, Cm, dy, skip=None, z=None, dt_bias=None, softplus=True, lengths=None, state=None, dstate_out=None):
    """Dict of the gradients of u, dt, A, Bm, Cm, skip, z, dt_bias and state."""
    B, L, D = u.shape
    N, G = A.shape[1], Bm.shape[2]
    _, _, all_h = scan_fwd(u, dt, A, Bm, Cm, skip, z, dt_bias, softplus, lengths, state, keep=True)
    g = {"u": np.zeros((B, L, D)), "dt": np.zeros((B, L, D)), "A": np.zeros((D, N)), "Bm": np.zeros((B, L, G, N)),
         "Cm": np.zeros((B, L, G, N)), "skip": np.zeros(D), "z": np.zeros((B, L, D)), "dt_bias": np.zeros(D),
         "state": np.zeros((B, D, N))}
    for b in range(B):
        n = L if lengths is None else int(lengths[b])
        dh = np.zeros((D, N)) if dstate_out is None else dstate_out[b].astype(np.float64)
        for t in range(n - 1, -1, -1):
            ut, d = u[b, t].astype(np.float64), dy[b, t].astype(np.float64)
            delta, raw = _delta(dt[b, t], dt_bias, softplus)
            bt, ct = (np.repeat(m[b, t].astype(np.float64), D // G, axis=0) for m in (Bm, Cm))
            before, h = all_h[b, t], all_h[b, t + 1]
            if z is not None:
                zt = z[b, t].astype(np.float64)
                y = (h * ct).sum(1) + (0 if skip is None else skip * ut)
                g["z"][b, t] = d * y * act_bwd(zt, True)
                d = d * act_fwd(zt, True)
            a = np.exp(delta[:, None] * A)
            dh = dh + d[:, None] * ct
            g["Cm"][b, t] = (d[:, None] * h).reshape(G, D // G, N).sum(1)
            g["Bm"][b, t] = (dh * (delta * ut)[:, None]).reshape(G, D // G, N).sum(1)
            grown = (dh * bt).sum(1)
            q = dh * a * before
            g["A"] += q * delta[:, None]
            ddelta = (q * A).sum(1) + grown * ut
            g["u"][b, t] = grown * delta + (0 if skip is None else skip * d)
            g["skip"] += d * ut
            g["dt"][b, t] = ddelta * (sigmoid(raw) if softplus else 1)
            g["dt_bias"] += g["dt"][b, t]
            dh = dh * a
        g["state"][b] = dh
    return g


# ---- linear attention ------------------------------------------------------------------------


def _log_decays(g, decay, b, n, H):
    ld = np.zeros((n, H))
    if g is not None:
        ld = ld + g[b, :n].astype(np.float64)
    if decay is not None:
        ld = ld + decay.astype(np.float64)
    return ld


def attention_fwd(q, k, v, scale, g=None, decay=None, lengths=None, state=None, keep=False):
    """(y, new state): q, k (B, L, Hk, Dk), v (B, L, H, Dv), g (B, L, H), decay (H), state (B, H, Dk, Dv).  keep: also
    every token's state."""
    B, L, H, Dv = v.shape
    shared, Dk = H // q.shape[2], q.shape[3]
    y, out = np.zeros((B, L, H, Dv)), np.zeros((B, H, Dk, Dv))
    all_s = np.zeros((B, L + 1, H, Dk, Dv)) if keep else None
    for b in range(B):
        n = L if lengths is None else int(lengths[b])
        ld = _log_decays(g, decay, b, n, H)
        s = np.zeros((H, Dk, Dv)) if state is None else state[b].astype(np.float64)
        if keep:
            all_s[b, 0] = s
        for t in range(n):
            qt, kt = (np.repeat(m[b, t].astype(np.float64), shared, axis=0) for m in (q, k))
            s = np.exp(ld[t])[:, None, None] * s + kt[:, :, None] * v[b, t].astype(np.float64)[:, None, :]
            y[b, t] = scale * (qt[:, :, None] * s).sum(1)
            if keep:
                all_s[b, t + 1] = s
        out[b] = s
    return (y, out, all_s) if keep else (y, out)


def attention_bwd(q, k, v, scale, dy, g=None, decay=None, lengths=None, state=None, dstate_out=None):
    """Dict of the gradients of q, k, v, g (of the log decays) and state."""
    B, L, H, Dv = v.shape
    Hk, Dk = q.shape[2:]
    shared = H // Hk
    _, _, all_s = attention_fwd(q, k, v, scale, g, decay, lengths, state, keep=True)
    out = {"q": np.zeros((B, L, Hk, Dk)), "k": np.zeros((B, L, Hk, Dk)), "v": np.zeros((B, L, H, Dv)), "g": np.zeros((B, L, H)),
           "state": np.zeros((B, H, Dk, Dv))}
    for b in range(B):
        n = L if lengths is None else int(lengths[b])
        ld = _log_decays(g, decay, b, n, H)
        ds = np.zeros((H, Dk, Dv)) if dstate_out is None else dstate_out[b].astype(np.float64)
        for t in reversed(range(n)):
            qt, kt = (np.repeat(m[b, t].astype(np.float64), shared, axis=0) for m in (q, k))
            vt, dyt = v[b, t].astype(np.float64), dy[b, t].astype(np.float64)
            ds = ds + scale * qt[:, :, None] * dyt[:, None, :]
            out["q"][b, t] = (scale * (all_s[b, t + 1] * dyt[:, None, :]).sum(2)).reshape(Hk, shared, Dk).sum(1)
            out["k"][b, t] = (ds * vt[:, None, :]).sum(2).reshape(Hk, shared, Dk).sum(1)
            out["v"][b, t] = (ds * kt[:, :, None]).sum(1)
            ds = np.exp(ld[t])[:, None, None] * ds
            out["g"][b, t] = (ds * all_s[b, t]).sum((1, 2))
        out["state"][b] = ds
    return out


# ---- gated projection ------------------------------------------------------------------------


def gate_act(v, act):
    """act(v), and its derivative; 0: none, 1: SiLU, 2: GELU in its tanh form, v sigmoid(2 sqrt(2/pi) (v + 0.044715 v^3))."""
    if act == 0:
        return v, np.ones_like(v)
    if act == 1:
        return act_fwd(v, True), act_bwd(v, True)
    c = 2 * np.sqrt(2 / np.pi)
    s = sigmoid(c * (v + 0.044715 * v ** 3))
    return v * s, s * (1 + v * (1 - s) * c * (1 + 3 * 0.044715 * v * v))


def gated_fwd(x, w_gate, w_up, act):
    x, w_gate, w_up = (a.astype(np.float64) for a in (x, w_gate, w_up))
    return gate_act(x @ w_gate.T, act)[0] * (x @ w_up.T)


def gated_bwd(x, w_gate, w_up, act, dy):
    """(dx, dw_gate, dw_up)."""
    x, w_gate, w_up, dy = (a.astype(np.float64) for a in (x, w_gate, w_up, dy))
    value, slope = gate_act(x @ w_gate.T, act)
    dgate, dup = dy * (x @ w_up.T) * slope, dy * value
    return dgate @ w_gate + dup @ w_up, dgate.T @ x, dup.T @ x
