"""Optimizer of the coefficient values: plain fp64 reference.

TEST INFRASTRUCTURE ONLY (same rules as frameft_oracle: only tests/, smoke() and
bench.py's cpu_baseline may use it; it shares nothing with the HIP library).

The paper trains only the coefficient values of C with AdamW under a linear
learning-rate schedule with warmup (Appendix G, the hyperparameter tables of the
GLUE, image-classification and instruction-tuning experiments).  AdamW is Adam
with the weight decay decoupled from the gradient (Loshchilov and Hutter,
"Decoupled Weight Decay Regularization"): the decay shrinks the parameters
directly instead of being added to the gradient.  The steps below follow that
algorithm in the order common training frameworks use: decay with the step's
learning rate, then the bias-corrected Adam step.  The schedule is the usual
linear warmup from 0 to the base rate over the warmup steps, then linear decay
to 0 at the last step.
"""
from __future__ import annotations

import math

import numpy as np


def adamw_step(c, g, m, v, t, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0):
    """One AdamW step at step number t (1 for the first step) on fp64 copies of the arrays.

    Returns (c, m, v) after the step:
        c <- c (1 - lr * weight_decay)                      (decoupled decay)
        m <- beta1 m + (1 - beta1) g                        (first moment)
        v <- beta2 v + (1 - beta2) g^2                      (second moment)
        c <- c - lr * (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
    """
    if t < 1:
        raise ValueError("step numbers start at 1")
    c = np.asarray(c, dtype=np.float64) * (1.0 - lr * weight_decay)
    g = np.asarray(g, dtype=np.float64)
    m = beta1 * np.asarray(m, dtype=np.float64) + (1.0 - beta1) * g
    v = beta2 * np.asarray(v, dtype=np.float64) + (1.0 - beta2) * g * g
    m_hat = m / (1.0 - beta1 ** t)
    v_hat = v / (1.0 - beta2 ** t)
    c = c - lr * m_hat / (np.sqrt(v_hat) + eps)
    return c, m, v


def warmup_steps(total_steps: int, warmup_ratio: float) -> int:
    """Warmup length for a ratio of the run (the tables give ratios 0.06 and 0.03), rounded up."""
    return int(math.ceil(total_steps * warmup_ratio))


def linear_warmup_lr(step: int, warmup: int, total: int, base_lr: float) -> float:
    """Learning rate of optimizer step `step` (0 for the first): rises linearly from 0 over
    `warmup` steps to base_lr, then falls linearly to 0 at step `total`."""
    if step < warmup:
        return base_lr * step / max(1, warmup)
    return base_lr * max(0.0, (total - step) / max(1, total - warmup))


# ------------------------------------------------------------------ moments of 8 bits

BLOCK = 256


def code_units(signed):
    """Units that each code without sign stands for: 128 of m, 256 of v."""
    return np.array([a if a < 16 else (8 + a % 8) * 2.0 ** (a // 8 - 1) for a in range(128 if signed else 256)])


def state_values(codes, exps, signed):
    """Values of codes (uint8) whose blocks of 256 have the stored exponents exps."""
    codes = np.asarray(codes).astype(np.int64)
    a = code_units(signed)[codes % 128 if signed else codes]
    a = np.where(codes >= 128, -a, a) if signed else a
    return a * np.repeat(2.0 ** (np.asarray(exps).astype(np.float64) - 120), BLOCK)[:codes.size]


def state_codes(x, h, signed):
    """(codes, exponents) of moments x (fp64, finite) with the 16 random bits h of each element.  Each block's unit is the least
    power of two (at least 2^-120) whose largest code reaches the block's largest value in fp32."""
    x, grid = np.asarray(x, dtype=np.float64), code_units(signed)
    codes, exps = np.zeros(x.size, dtype=np.uint8), np.zeros(-(-x.size // BLOCK), dtype=np.uint8)
    for b in range(exps.size):
        s = slice(b * BLOCK, min(x.size, (b + 1) * BLOCK))
        most = float(np.float32(np.abs(x[s]).max()))
        k = -120
        while most > grid[-1] * 2.0 ** k:
            k += 1
        y = np.abs(x[s]) / 2.0 ** k
        at = np.minimum(np.searchsorted(grid, y, side="right") - 1, grid.size - 2)
        share = (y - grid[at]) / (grid[at + 1] - grid[at])
        a = at + (share + (h[s] + 0.5) / 65536.0 >= 1.0)
        a = np.where((x[s] < 0), a + 128, a) if signed else np.where((a == 0) & (x[s] > 0), 1, a)
        codes[s], exps[b] = a, k + 120
    return codes, exps


def state_draws(n, step, tensor, seed):
    """The 16 random bits of (m, v) of each of n elements: Philox 4x32-10 (train_oracle.philox4x32) of (element / 4, step,
    tensor) under seed; element i takes word i % 4, m its low half."""
    from .train_oracle import philox4x32
    b = np.arange(-(-n // 4), dtype=np.uint64)
    c = np.stack([b & np.uint64(0xFFFFFFFF), b >> np.uint64(32), np.full_like(b, step % 2 ** 32), np.full_like(b, tensor)], axis=-1)
    w = philox4x32(c, (seed % 2 ** 32, seed // 2 ** 32)).reshape(-1)[:n].astype(np.int64)
    return w % 65536, w // 65536


def adamw8_step(c, g, m, v, mx, vx, t, tensor, seed, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0):
    """adamw_step with 8-bit moments: codes m, v (uint8) with exponents mx, vx.  Returns (c, m, v, mx, vx), c in fp64."""
    n = np.asarray(c).size
    c1, m1, v1 = adamw_step(c, g, state_values(m, mx, True), state_values(v, vx, False), t, lr, beta1, beta2, eps, weight_decay)
    top = float(np.finfo(np.float32).max)
    keep = (np.abs(m1) <= top) & (v1 <= top)
    m1, v1 = np.where(keep, m1, 0.0), np.where(keep, v1, 0.0)
    hm, hv = state_draws(n, t, tensor, seed)
    m2, mx2 = state_codes(m1, hm, True)
    v2, vx2 = state_codes(v1, hv, False)
    return c1, m2, v2, mx2, vx2
