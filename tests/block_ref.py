"""Plain float64 forms of the operators over packed sequences, token by token, for the tests.

Each takes ``mag=True`` for its majorant: the same sums over the operands' absolute values (decays and activations as they
are).  Rounding errors of the kernels are bounded by a factor times that, however much the true sums cancel.
"""
import numpy as np


def sigmoid(u):
    return 0.5 * (1.0 + np.tanh(0.5 * np.asarray(u, dtype=np.float64)))


def silu(u):
    return u * sigmoid(u)


def d_silu(u):
    s = sigmoid(u)
    return s * (1.0 + u * (1.0 - s))


def softplus(u):
    return np.maximum(u, 0.0) + np.log1p(np.exp(-np.abs(u)))


def offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def conv(x, w, bias, lengths, state=None, act=True):
    """(y, state_out); rows behind the last sequence are zero in y."""
    W, D = w.shape[1], x.shape[1]
    y, states, at = np.zeros(x.shape), [], 0
    for s, n in enumerate(lengths):
        head = np.zeros((W - 1, D)) if state is None else state[s]
        ext = np.concatenate([head, x[at:at + n]]).astype(np.float64)
        for t in range(n):
            u = np.zeros(D) if bias is None else bias.astype(np.float64)
            for j in range(W):
                u = u + w[:, j] * ext[W - 1 + t - j]
            y[at + t] = silu(u) if act else u
        states.append(ext[n:n + W - 1])
        at += n
    return y, np.array(states).reshape(len(lengths), W - 1, D)


def conv_bwd(x, w, bias, d_y, lengths, state=None, d_state_out=None, act=True, mag=False):
    """(d_x, d_w, d_bias, d_state_in)"""
    f = np.abs if mag else (lambda v: v)
    W, D = w.shape[1], x.shape[1]
    d_x, d_w, d_b, d_s, at = np.zeros(x.shape), np.zeros((D, W)), np.zeros(D), [], 0
    for s, n in enumerate(lengths):
        head = np.zeros((W - 1, D)) if state is None else state[s]
        ext = np.concatenate([head, x[at:at + n]]).astype(np.float64)
        d_ext = np.zeros(ext.shape)
        if d_state_out is not None:
            d_ext[n:] += f(d_state_out[s])
        for t in range(n):
            u = np.zeros(D) if bias is None else bias.astype(np.float64)
            for j in range(W):
                u = u + w[:, j] * ext[W - 1 + t - j]
            du = f(d_y[at + t] * (d_silu(u) if act else 1.0))
            if mag and act:   # the slope's own error: it changes by at most 0.5 per unit of u, u is off by roundings of its terms
                du = du + np.abs(d_y[at + t]) * (1.0 + sum(np.abs(w[:, j] * ext[W - 1 + t - j]) for j in range(W)))
            d_b += du
            for j in range(W):
                d_w[:, j] += du * f(ext[W - 1 + t - j])
                d_ext[W - 1 + t - j] += f(w[:, j]) * du
        d_x[at:at + n] = d_ext[W - 1:]
        d_s.append(d_ext[:W - 1])
        at += n
    return d_x, d_w, d_b, np.array(d_s).reshape(len(lengths), W - 1, D)


def _groups(v, D):
    return np.repeat(v, D // v.shape[0], axis=0)


def scan(x, dt, a, b, c, lengths, d_skip=None, z=None, dt_bias=None, soft=True, state=None, mag=False):
    """(y, state_out)"""
    f = np.abs if mag else (lambda v: v)
    D, N = a.shape
    raw = dt.astype(np.float64) + (0.0 if dt_bias is None else dt_bias)
    step = softplus(raw) if soft else raw
    y, states, at = np.zeros(x.shape), [], 0
    for s, n in enumerate(lengths):
        h = np.zeros((D, N)) if state is None else f(state[s].astype(np.float64))
        for t in range(at, at + n):
            h = np.exp(step[t][:, None] * a) * h + f(step[t] * x[t])[:, None] * f(_groups(b[t], D))
            y[t] = (h * f(_groups(c[t], D))).sum(1) + (0.0 if d_skip is None else f(d_skip * x[t]))
            if z is not None:
                y[t] *= f(silu(z[t].astype(np.float64)))
        states.append(h)
        at += n
    return y, np.array(states)


def scan_bwd(x, dt, a, b, c, d_y, lengths, d_skip=None, z=None, dt_bias=None, soft=True, state=None, d_state_out=None, mag=False):
    """dict of the gradients"""
    f = np.abs if mag else (lambda v: v)
    T, D = x.shape
    N, G = a.shape[1], b.shape[1]
    raw = dt.astype(np.float64) + (0.0 if dt_bias is None else dt_bias)
    step = softplus(raw) if soft else raw
    slope = sigmoid(raw) if soft else np.ones_like(raw)
    g = {k: np.zeros(x.shape) for k in ("d_x", "d_dt", "d_z")}
    g |= {k: np.zeros(b.shape) for k in ("d_b", "d_c")}
    g |= {"d_a": np.zeros((D, N)), "d_skip": np.zeros(D), "d_dt_bias": np.zeros(D), "d_state_in": []}
    at = 0
    for s, n in enumerate(lengths):
        h = np.zeros((D, N)) if state is None else f(state[s].astype(np.float64))
        hs = [h]
        for t in range(at, at + n):
            h = np.exp(step[t][:, None] * a) * h + f(step[t] * x[t])[:, None] * f(_groups(b[t], D))
            hs.append(h)
        e = np.zeros((D, N)) if d_state_out is None else f(d_state_out[s].astype(np.float64))
        for t in range(at + n - 1, at - 1, -1):
            h, prev = hs[t - at + 1], hs[t - at]
            bt, ct = f(_groups(b[t], D)), f(_groups(c[t], D))
            gate = 1.0 if z is None else f(silu(z[t].astype(np.float64)))
            pre = (h * ct).sum(1) + (0.0 if d_skip is None else f(d_skip * x[t]))
            if z is not None:
                g["d_z"][t] = f(d_y[t]) * pre * f(d_silu(z[t].astype(np.float64)))
                if mag:
                    g["d_z"][t] += np.abs(d_y[t]) * pre
            dg = f(d_y[t] * gate)
            gh = ct * dg[:, None] + e
            decay = np.exp(step[t][:, None] * a)
            e = decay * gh
            g_b = (gh * bt).sum(1)
            through = e * prev
            g["d_c"][t] = (dg[:, None] * h).reshape(G, D // G, N).sum(1)
            g["d_b"][t] = (gh * f(step[t] * x[t])[:, None]).reshape(G, D // G, N).sum(1)
            g["d_dt"][t] = ((through * f(a)).sum(1) + f(x[t]) * g_b) * slope[t]
            g["d_x"][t] = f(step[t]) * g_b + (0.0 if d_skip is None else f(d_skip) * dg)
            g["d_a"] += through * f(step[t])[:, None]
            g["d_skip"] += dg * f(x[t])
            g["d_dt_bias"] += g["d_dt"][t]
        g["d_state_in"].append(e)
        at += n
    g["d_state_in"] = np.array(g["d_state_in"])
    return g


def act_fn(kind):
    return {0: lambda u: u, 1: silu, 2: sigmoid}[kind]


def d_act_fn(kind):
    return {0: lambda u: np.ones_like(u), 1: d_silu, 2: lambda u: sigmoid(u) * (1 - sigmoid(u))}[kind]


def normalised(v, kind, eps):
    """(normalised rows, 1 / deviation) for kind 0 none, 1 rms, 2 layer"""
    if kind == 0:
        return v, np.ones((v.shape[0], 1))
    if kind == 2:
        v = v - v.mean(1, keepdims=True)
    inv = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return v * inv, inv


def norm_back(d, hat, inv, kind):
    if kind == 0:
        return d
    r = d - hat * (d * hat).mean(1, keepdims=True)
    return inv * (r - d.mean(1, keepdims=True) if kind == 2 else r)


def junction(res, y, gate, w_post, b_post, norm_post, scale, w_pre, b_pre, norm_pre, gate_act, gate_after, eps):
    """(r', o) and what the backward pass wants"""
    keep = {}
    r = 0.0 if res is None else res.astype(np.float64)
    if y is not None:
        y = y.astype(np.float64)
        ga = np.ones_like(y) if gate is None else act_fn(gate_act)(gate.astype(np.float64))
        hat, inv = normalised(y if gate_after else y * ga, norm_post, eps)
        n = hat * (1.0 if w_post is None else w_post) + (0.0 if b_post is None else b_post)
        m = n * ga if gate_after else n
        r = r + (1.0 if scale is None else scale) * m
        keep = {"y": y, "ga": ga, "hat": hat, "inv": inv, "n": n, "m": m}
    hat2, inv2 = normalised(r, norm_pre, eps)
    return r, hat2 * (1.0 if w_pre is None else w_pre) + (0.0 if b_pre is None else b_pre), keep


def junction_bwd(r, y, gate, d_o, d_r, w_post, b_post, norm_post, scale, w_pre, b_pre, norm_pre, gate_act, gate_after, eps):
    """dict of the gradients, from r' as it is given"""
    D = r.shape[1]
    zero = np.zeros(r.shape)
    g = {k: np.zeros(D) for k in ("d_w_post", "d_b_post", "d_scale", "d_w_pre", "d_b_pre")}
    d = zero if d_r is None else d_r.astype(np.float64)
    if d_o is not None:
        d_o = d_o.astype(np.float64)
        hat2, inv2 = normalised(r.astype(np.float64), norm_pre, eps)
        g["d_w_pre"], g["d_b_pre"] = (d_o * hat2).sum(0), d_o.sum(0)
        d = d + norm_back(d_o * (1.0 if w_pre is None else w_pre), hat2, inv2, norm_pre)
    g["d_res"] = d
    if y is not None:
        _, _, k = junction(None, y, gate, w_post, b_post, norm_post, scale, None, None, 0, gate_act, gate_after, eps)
        d_m = d * (1.0 if scale is None else scale)
        g["d_scale"] = (d * k["m"]).sum(0)
        d_n = d_m * k["ga"] if gate_after else d_m
        g["d_w_post"], g["d_b_post"] = (d_n * k["hat"]).sum(0), d_n.sum(0)
        d_v = norm_back(d_n * (1.0 if w_post is None else w_post), k["hat"], k["inv"], norm_post)
        g["d_y"] = d_v if gate_after else d_v * k["ga"]
        if gate is not None:
            g["d_gate"] = (d_m * k["n"] if gate_after else d_v * k["y"]) * d_act_fn(gate_act)(gate.astype(np.float64))
    return g
