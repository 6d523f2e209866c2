"""The rms norm with the residual's addition, dropout's counter, the choice of key
blocks and the attention over chosen blocks in fp64, with their backward passes. TEST
INFRASTRUCTURE ONLY (see the package docstring).

Rms norm of rows h (.., D): r = 1/sqrt(mean h^2 + eps), n = h r, y = n w; with g = dy w
the gradients are dh = r (g - n mean(g n)), dw = sum dy n.

Dropout: element c of row r is kept if its sixteen bits are at least round(65536 p):
half c % 8 of the four words of Philox 4x32 (ten rounds) for the counter (c / 8, r, offset)
and the key `seed`.
"""
from __future__ import annotations

import math

import numpy as np

MASK = np.uint64(0xffffffff)


def philox(counter, key):
    """Four 32-bit words (.., 4) for counters (.., 4) and keys (.., 2)."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [np.asarray(key[..., i], dtype=np.uint64) for i in range(2)]
    for _ in range(10):
        x, y = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(y >> np.uint64(32)) ^ c[1] ^ k[0], y & MASK, (x >> np.uint64(32)) ^ c[3] ^ k[1], x & MASK]
        k = [(k[0] + np.uint64(0x9E3779B9)) & MASK, (k[1] + np.uint64(0xBB67AE85)) & MASK]
    return np.stack(c, -1)


def kept(shape, p, seed, offset):
    """Which elements of an array of this shape stay, and what these are multiplied with."""
    D, rows = shape[-1], math.prod(shape[:-1])
    n = -(-D // 8)
    c = np.zeros((rows, n, 4), dtype=np.uint64)
    c[..., 0], c[..., 1] = np.arange(n), np.arange(rows)[:, None]
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    c[..., 2], c[..., 3] = offset & 0xffffffff, offset >> 32
    w = philox(c, np.array([seed & 0xffffffff, seed >> 32], dtype=np.uint64))
    half = np.stack((w & np.uint64(0xffff), w >> np.uint64(16)), -1).reshape(rows, n * 8)[:, :D]
    t = round(p * 65536)
    return (half >= t).reshape(shape), 65536.0 / (65536 - t) if t < 65536 else 0.0


def rms_norm(h, w, eps):
    """h (.., D), w (D) or None -> y, r."""
    h = np.asarray(h, dtype=np.float64)
    r = 1.0 / np.sqrt((h * h).mean(-1) + eps)
    y = h * r[..., None]
    return (y if w is None else y * w), r


def rms_norm_backward(h, w, eps, dy):
    """The gradients dh and dw for the upstream gradient dy."""
    h, dy = np.asarray(h, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    n, r = rms_norm(h, None, eps)
    g = dy if w is None else dy * w
    return r[..., None] * (g - n * (g * n).mean(-1, keepdims=True)), (dy * n).sum(tuple(range(h.ndim - 1)))


def _eighths(mean):
    mean = np.where(np.isfinite(mean), mean, 0.0)
    top = np.abs(mean).max(-1)
    by = np.where(top > 0, 127.0 * (1.0 / np.where(top > 0, top, 1.0)), 0.0)
    return np.rint(mean * by[..., None]), top


def block_means(k, block, key_lens=None):
    """k (B, Hk, Nk, d) -> whole numbers (B, Hk, blocks, d) and scales (B, Hk, blocks), -1 of a block without keys."""
    B, Hk, Nk, d = k.shape
    nb = -(-Nk // block)
    m, scale = np.zeros((B, Hk, nb, d)), np.full((B, Hk, nb), -1.0, dtype=np.float32)
    for b in range(B):
        n = Nk if key_lens is None else min(max(int(key_lens[b]), 0), Nk)
        for j in range(-(-n // block)):
            part = np.asarray(k[b, :, j * block:min(n, (j + 1) * block)], dtype=np.float64)
            m[b, :, j], top = _eighths(part.sum(1) / part.shape[1])
            scale[b, :, j] = (top * (1.0 / 127.0)).astype(np.float32)
    return m, scale


def block_select(q, means, topk, q_block):
    """The topk blocks (B, H, groups, topk) of highest score in ascending order, then -1."""
    m, scale = means
    B, H, Nq, d = q.shape
    Hk, nb = m.shape[1:3]
    groups = -(-Nq // q_block)
    out = np.full((B, H, groups, topk), -1, dtype=np.int32)
    for b in range(B):
        for h in range(H):
            hk = h // (H // Hk)
            x = np.stack([np.asarray(q[b, h, g * q_block:(g + 1) * q_block], dtype=np.float64).sum(0)
                          / min(q_block, Nq - g * q_block) for g in range(groups)])
            x, _ = _eighths(x)
            score = (x @ m[b, hk].T).astype(np.float32) * scale[b, hk]
            for g in range(groups):
                there = np.flatnonzero(scale[b, hk] >= 0)
                best = sorted(there, key=lambda j: (-score[g, j], j))[:topk]
                out[b, h, g, :len(best)] = sorted(best)
    return out


def allowed(blocks, Nq, Nk, block, q_block, key_lens=None):
    """Which keys (B, H, Nq, Nk) each query attends to."""
    B, H, groups, _ = blocks.shape
    nb = -(-Nk // block)
    hit = np.zeros((B, H, groups, nb), dtype=bool)
    for j in range(nb):
        hit[..., j] = (blocks == j).any(-1)
    mask = hit[:, :, np.arange(Nq) // q_block][..., np.arange(Nk) // block]
    if key_lens is not None:
        mask &= (np.arange(Nk) < np.asarray(key_lens)[:, None])[:, None, None]
    return mask


def block_attention(q, k, v, mask, scale, dout=None):
    """q (B, H, Nq, d), k and v (B, Hk, Nk, d), mask from `allowed`: a dict of o, o32 and lse,
    and with dout of dq, dk and dv. Under the same names with "_off" stands a bound of what
    the rounding to bf16 of P and dS (as operands) and of the outputs can change, half a step
    (2^-8) each, with fp32 sums. Keys and values outside the mask are not read."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    B, H, Nq, d = q.shape
    Hk, Nk = k.shape[1:3]
    u = 2.0 ** -8
    r = {n: np.zeros((B, H, Nq, d)) for n in ("o", "o32", "o_off", "o32_off")}
    r["lse"], r["lse_off"] = np.full((B, H, Nq), -np.inf), np.zeros((B, H, Nq))
    if dout is not None:
        dout = np.asarray(dout, dtype=np.float64)
        for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", v.shape)):
            r[n], r[n + "_off"] = np.zeros(s), np.zeros(s)
    for b in range(B):
        for h in range(H):
            hk, M = h // (H // Hk), mask[b, h]
            rows, used = M.any(1), M.any(0)
            if not rows.any():
                continue
            kk, vv = np.where(used[:, None], k[b, hk], 0.0), np.where(used[:, None], v[b, hk], 0.0)
            s = np.where(M, scale * q[b, h] @ kk.T, -np.inf)
            top = np.where(rows, s.max(1), 0.0)[:, None]
            e = np.exp(s - top)
            tot = e.sum(1, keepdims=True)
            P = np.where(rows[:, None], e / np.where(rows[:, None], tot, 1.0), 0.0)
            O, A = P @ vv, P @ np.abs(vv)
            lse = np.where(rows, (top + np.log(np.where(rows[:, None], tot, 1.0)))[:, 0], -np.inf)
            r["lse"][b, h] = lse
            size = scale * np.where(M, np.abs(q[b, h]) @ np.abs(kk).T, 0.0).max(1)
            off = np.where(rows, 2.0 ** -24 * (d + 16) * size + 2.0 ** -22 * np.abs(np.where(rows, lse, 0.0)) + 2e-6, 0.0)
            r["lse_off"][b, h] = off
            fp32 = 2.0 ** -24 * (d + 64) * (1 + off.max() * 2.0 ** 24 / (d + 64))
            o_in = (u + fp32) * A
            r["o32"][b, h], r["o32_off"][b, h] = O, o_in
            r["o"][b, h], r["o_off"][b, h] = O, o_in + u * (np.abs(O) + o_in)
            if dout is None:
                continue
            g = dout[b, h]
            r["dv"][b, hk] += P.T @ g
            r["dv_off"][b, hk] += (u + fp32) * P.T @ np.abs(g)
            dP, D = g @ vv.T, (g * O).sum(1, keepdims=True)
            D_off = (np.abs(g) * o_in).sum(1, keepdims=True)
            ds = P * (dP - D)
            ds_off = u * np.abs(ds) + (1 + u) * P * D_off + fp32 * P * (np.abs(g) @ np.abs(vv).T + np.abs(D))
            dq, dq_in = scale * ds @ kk, scale * ds_off @ np.abs(kk)
            r["dq"][b, h], r["dq_off"][b, h] = dq, dq_in + u * (np.abs(dq) + dq_in)
            r["dk"][b, hk] += scale * ds.T @ q[b, h]
            r["dk_off"][b, hk] += scale * ds_off.T @ np.abs(q[b, h])
    if dout is not None:
        for n in ("dk", "dv"):
            r[n + "_off"] += u * (np.abs(r[n]) + r[n + "_off"])
    return r
