"""Layer norm, rotary positions with several axes and differential attention in
fp64, each with its backward pass. TEST INFRASTRUCTURE ONLY (see the package
docstring).

Layer norm of rows x (.., D): mu = mean x, r = 1/sqrt(var x + eps),
h = (x - mu) r, y = h w + b; with g = dy w the gradients are
dx = r (g - mean g - h mean(g h)), dw = sum dy h, db = sum dy.

Rotary positions: pair p turns by position times frequency, see `rotary`.

Differential attention, per head with two maps of queries and keys and one set
of values: P_m = softmax(scale Q_m K_m^T), O = P_1 V - lam P_2 V.
"""
from __future__ import annotations

import numpy as np


def layer_norm(x, w, b, eps):
    """x (.., D), w and b (D) or None -> y, mean, rstd."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    dev = x - mean[..., None]
    rstd = 1.0 / np.sqrt((dev * dev).mean(-1) + eps)
    y = dev * rstd[..., None]
    if w is not None:
        y = y * w
    if b is not None:
        y = y + b
    return y, mean, rstd


def layer_norm_backward(x, w, eps, dy):
    """The gradients dx, dw, db for the upstream gradient dy."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    h, _, rstd = layer_norm(x, None, None, eps)
    g = dy if w is None else dy * w
    dx = rstd[..., None] * (g - g.mean(-1, keepdims=True) - h * (g * h).mean(-1, keepdims=True))
    rows = tuple(range(x.ndim - 1))
    return dx, (dy * h).sum(rows), dy.sum(rows)


def rotary_angles(positions, sections, base, joint=False):
    """Angles (.., R) of positions (.., A): pair i of the n of an axis turns by
    its position times base^(-i/n); joint: pair p of all R by base^(-p/R)."""
    positions = np.asarray(positions, dtype=np.float64)
    R = sum(sections)
    cols, p = [], 0
    for a, n in enumerate(sections):
        for i in range(n):
            cols.append(positions[..., a] * float(base) ** -(p / R if joint else i / n))
            p += 1
    return np.stack(cols, -1)


def rotary(x, positions, sections, base, interleaved=False, joint=False, inverse=False):
    """x (B, H, N, d), positions (N, A) or (B, N, A): (a, b) of a pair becomes
    (a cos - b sin, b cos + a sin). Pairs are columns (p, R + p), or (2p, 2p + 1)
    if interleaved."""
    y = np.array(x, dtype=np.float64)
    t = rotary_angles(positions, sections, base, joint)
    t = t[:, None] if t.ndim == 3 else t
    if inverse:
        t = -t
    R = sum(sections)
    lo, hi = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
    a, b = y[..., lo].copy(), y[..., hi].copy()
    y[..., lo] = a * np.cos(t) - b * np.sin(t)
    y[..., hi] = b * np.cos(t) + a * np.sin(t)
    return y


def _softmax(s):
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    tot = e.sum(-1, keepdims=True)
    return e / tot, (m + np.log(tot))[..., 0]


def diff_attention(q, k, v, lam, scale, key_lens=None, dout=None):
    """q (B, 2H, Nq, d), k (B, 2H, Nk, d), v (B, H, Nk, e), lam (H): a dict of o,
    o2 (B, 2H, Nq, e: each map's output) and lse (B, 2H, Nq), and with dout of dq,
    dk, dv and dlam. Under the same names with "_off" stands a bound of what the
    rounding to bf16 of P and dS (as operands) and of the outputs can change, half a
    step (2^-8) each, with fp32 sums."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    B, H, Nk, e = v.shape
    Nq, d = q.shape[2], q.shape[3]
    u = 2.0 ** -8
    r = {"o": np.zeros((B, H, Nq, e)), "o2": np.zeros((B, 2 * H, Nq, e)), "lse": np.full((B, 2 * H, Nq), -np.inf),
         "o_off": np.zeros((B, H, Nq, e)), "o2_off": np.zeros((B, 2 * H, Nq, e)), "lse_off": np.zeros((B, 2 * H, Nq))}
    if dout is not None:
        dout = np.asarray(dout, dtype=np.float64)
        for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", v.shape), ("dlam", (H,))):
            r[n], r[n + "_off"] = np.zeros(s), np.zeros(s)
    for b in range(B):
        n = Nk if key_lens is None else int(key_lens[b])
        if n == 0:
            continue
        for h in range(H):
            vv, la, P, O, A = v[b, h, :n], float(lam[h]), [], [], []
            for m in (0, 1):
                s = scale * q[b, 2 * h + m] @ k[b, 2 * h + m, :n].T
                p, lse = _softmax(s)
                P.append(p)
                O.append(p @ vv)
                A.append(p @ np.abs(vv))
                r["lse"][b, 2 * h + m] = lse
                # fp32 sums of d products, and of the probabilities
                size = scale * (np.abs(q[b, 2 * h + m]) @ np.abs(k[b, 2 * h + m, :n]).T).max(-1)
                r["lse_off"][b, 2 * h + m] = 2.0 ** -24 * (d + 16) * size + 2.0 ** -22 * np.abs(lse) + 2e-6
            # the sum of the probabilities is of their unrounded values
            fp32 = 2.0 ** -24 * (d + 64) * (1 + r["lse_off"][b, 2 * h:2 * h + 2].max() * 2.0 ** 24 / (d + 64))
            o, o_in = O[0] - la * O[1], (u + fp32) * (A[0] + abs(la) * A[1])
            r["o"][b, h] = o
            r["o_off"][b, h] = o_in + u * (np.abs(o) + o_in)
            for m in (0, 1):
                r["o2"][b, 2 * h + m], r["o2_off"][b, 2 * h + m] = O[m], (u + fp32) * A[m]
            if dout is None:
                continue
            g = dout[b, h]
            dP = g @ vv.T
            off1, off2 = ((np.abs(g) * r["o2_off"][b, 2 * h + m]).sum(-1) for m in (0, 1))
            w = P[0] - la * P[1]
            dv, dv_in = w.T @ g, (u * np.abs(w) + fp32 * (P[0] + abs(la) * P[1])).T @ np.abs(g)
            r["dv"][b, h, :n] = dv
            r["dv_off"][b, h, :n] = dv_in + u * (np.abs(dv) + dv_in)
            for m, f, off in ((0, 1.0, off1), (1, -la, off2)):
                D = (g * O[m]).sum(-1)
                if m:
                    r["dlam"][h] -= D.sum()
                    r["dlam_off"][h] += off.sum()
                ds = P[m] * (dP - D[:, None])
                grow = fp32 * P[m] * (np.abs(g) @ np.abs(vv).T + np.abs(D)[:, None])
                ds_off = (2 * u + u * u) * np.abs(ds) + (1 + 2 * u) * P[m] * off[:, None] + grow
                c = scale * f
                for name, x, xo in (("dq", c * ds @ k[b, 2 * h + m, :n], abs(c) * ds_off @ np.abs(k[b, 2 * h + m, :n])),
                                    ("dk", c * ds.T @ q[b, 2 * h + m], abs(c) * ds_off.T @ np.abs(q[b, 2 * h + m]))):
                    at = (b, 2 * h + m) if name == "dq" else (b, 2 * h + m, slice(0, n))
                    r[name][at] = x
                    r[name + "_off"][at] = xo + u * (np.abs(x) + xo)
    if dout is not None:
        r["dlam_off"] += 2.0 ** -8 * (np.abs(r["dlam"]) + r["dlam_off"])
    return r
