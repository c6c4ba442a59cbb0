"""Layer norm, dropout and the head's cross entropy: plain fp64 references.

TEST INFRASTRUCTURE ONLY (same rules as frameft_oracle: only tests/ may use it; it shares nothing
with the HIP library).

Dropout's mask is that of the library's definition: Philox 4x32 with ten rounds (Salmon, Moraes,
Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), written here from the paper's
description and pinned by its published known answers.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ layer norm

def layernorm_fwd(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x, variance over n."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1)
    xc = x - mean[:, None]
    rstd = 1.0 / np.sqrt((xc * xc).mean(axis=1) + eps)
    y = xc * rstd[:, None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean, rstd


def layernorm_bwd(x, g, weight=None, eps=1e-5):
    """(dx, dweight, dbias) of sum(g * layernorm(x))."""
    x, g = np.asarray(x, dtype=np.float64), np.asarray(g, dtype=np.float64)
    h, _, rstd = layernorm_fwd(x, eps=eps)
    a = g if weight is None else g * weight
    dx = rstd[:, None] * (a - a.mean(axis=1, keepdims=True) - h * (a * h).mean(axis=1, keepdims=True))
    return dx, (g * h).sum(axis=0), g.sum(axis=0)


# ------------------------------------------------------------------ dropout

def philox4x32(counter, key, rounds=10):
    """Four uint32 words (an array (..., 4)) of Philox for counters (..., 4) under key (2 words)."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    m32 = np.uint64(0xFFFFFFFF)
    for _ in range(rounds):
        a = c[0] * np.uint64(0xD2511F53)
        b = c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, axis=-1).astype(np.uint32)


def dropout_draws(p):
    """D of the 65536 values of a draw that are dropped."""
    return 65536 if p >= 1 else min(int(np.rint(p * 65536.0)), 65535)


def dropout_mask(T, n, p, seed, offset=0):
    """T x n, true where an element is kept."""
    nb = (n + 7) // 8
    block = np.arange(T * nb, dtype=np.uint64)
    offset &= (1 << 64) - 1
    seed &= (1 << 64) - 1
    counter = np.empty((T * nb, 4), dtype=np.uint64)
    counter[:, 0] = block & np.uint64(0xFFFFFFFF)
    counter[:, 1] = block >> np.uint64(32)
    counter[:, 2] = offset & 0xFFFFFFFF
    counter[:, 3] = offset >> 32
    w = philox4x32(counter, (seed & 0xFFFFFFFF, seed >> 32)).astype(np.int64)
    draws = np.stack([w & 0xFFFF, w >> 16], axis=-1).reshape(T, nb * 8)[:, :n]
    return draws >= dropout_draws(p)


def dropout(x, p, seed, offset=0, residual=None):
    x = np.asarray(x, dtype=np.float64)
    keep = dropout_mask(x.shape[0], x.shape[1], p, seed, offset)
    d = dropout_draws(p)
    y = np.where(keep, x * (65536.0 / max(65536 - d, 1)), 0.0)
    return y if residual is None else y + residual


# ------------------------------------------------------------------ cross entropy of a head

def xent(H, W, target, dloss=None, scale=1.0, rows=64):
    """(loss, lse, dH, dW, absolute sums) of the tokens of H (T x n) against the vocabulary W (V x n);
    targets outside [0, V) have loss 0 and no gradient.  The absolute sums are those that error bounds
    need: zabs[t] = max_v sum_c |h_c w_vc|, dH_abs = |P| |W|, dW_abs = |P|^T |H| (H's skipped rows as
    zeros)."""
    H, W = np.asarray(H, dtype=np.float64), np.asarray(W, dtype=np.float64)
    T, V = H.shape[0], W.shape[0]
    target = np.asarray(target)
    counted = (target >= 0) & (target < V)
    up = np.where(counted, scale * (np.ones(T) if dloss is None else np.asarray(dloss, dtype=np.float64)), 0.0)
    loss, lse, zabs = np.zeros(T), np.empty(T), np.empty(T)
    dH, dW = np.zeros_like(H), np.zeros_like(W)
    dHa, dWa = np.zeros_like(H), np.zeros_like(W)
    Wa = np.abs(W)
    for t0 in range(0, T, rows):
        s = slice(t0, min(T, t0 + rows))
        with np.errstate(invalid="ignore"):
            z = H[s] @ W.T
            top = z.max(axis=1, keepdims=True)
            e = np.exp(z - top)
            lse[s] = top[:, 0] + np.log(e.sum(axis=1))
            zabs[s] = (np.abs(H[s]) @ Wa.T).max(axis=1)
        P = np.zeros_like(z)
        for i, t in enumerate(range(s.start, s.stop)):
            if counted[t]:
                loss[t] = lse[t] - z[i, target[t]]
                P[i] = np.exp(z[i] - lse[t])
                P[i, target[t]] = -np.delete(P[i], target[t]).sum()      # p - 1, without cancellation
                P[i] *= up[t]
        live = np.where(counted[s, None], H[s], 0.0)
        dH[s] = P @ W
        dW += P.T @ live
        dHa[s] = np.abs(P) @ Wa
        dWa += np.abs(P).T @ np.abs(live)
    return loss, lse, dH, dW, (zabs, dHa, dWa)


# ------------------------------------------------------------------ join of two blocks

def _norm(kind, v, eps):
    """(normalised rows, mean, 1 / deviation); zeros where there is no norm."""
    zero = np.zeros((v.shape[0], 1))
    if kind == "none":
        return v, zero, zero
    mean = v.mean(axis=1, keepdims=True) if kind == "layer" else zero
    rstd = 1.0 / np.sqrt(((v - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    return (v - mean) * rstd, mean, rstd


def _norm_grad(kind, h, rstd, a):
    d = a - h * (a * h).mean(axis=1, keepdims=True)
    return rstd * (d - a.mean(axis=1, keepdims=True) if kind == "layer" else d)


def resnorm(r, b, gate=None, post="none", pw=None, pb=None, norm="rms", w=None, bias=None, res=1.0, block=1.0, eps=1e-5,
            dx=None, dy=None):
    """The join x = res r + block gate post(b), y = norm(x) and, from dx and dy, its backward.  gate: None, n elements or rows of n
    for equal shares of the rows.  Returns a dict with all values and, with dx or dy, all gradients."""
    r, b = np.asarray(r, dtype=np.float64), np.asarray(b, dtype=np.float64)
    T, n = r.shape
    one, zero = np.ones(n), np.zeros(n)
    pw, w = (one if v is None else np.asarray(v, dtype=np.float64) for v in (pw, w))
    pb, bias = (zero if v is None else np.asarray(v, dtype=np.float64) for v in (pb, bias))
    g = np.ones((1, n)) if gate is None else np.atleast_2d(np.asarray(gate, dtype=np.float64))
    rows = T // g.shape[0]
    G = np.repeat(g, rows, axis=0)
    o = dict(G=G, pw=pw, w=w, pb=pb, bias=bias)
    o["hp"], o["mp"], o["rp"] = _norm(post, b, eps)
    o["p"] = o["hp"] * pw + pb if post != "none" else b
    o["x"] = res * r + block * G * o["p"]
    o["h"], o["m"], o["q"] = _norm(norm, o["x"], eps)
    if norm != "none":
        o["y"] = o["h"] * w + bias
    if dx is None and dy is None:
        return o
    D = np.zeros((T, n)) if dx is None else np.asarray(dx, dtype=np.float64)
    if norm != "none":
        dy = np.asarray(dy, dtype=np.float64)
        D = D + _norm_grad(norm, o["h"], o["q"], dy * w)
        o["dw"], o["dbias"] = (dy * o["h"]).sum(axis=0), dy.sum(axis=0)
    o["D"], o["dr"], o["e"] = D, res * D, block * G * D
    o["dgate"] = (block * D * o["p"]).reshape(g.shape[0], rows, n).sum(axis=1)
    o["db"] = o["e"]
    if post != "none":
        o["dpw"], o["dpb"] = (o["e"] * o["hp"]).sum(axis=0), o["e"].sum(axis=0)
        o["db"] = _norm_grad(post, o["hp"], o["rp"], o["e"] * pw)
    return o
