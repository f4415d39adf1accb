"""The optimizer's side of a training step in binary64, on dense [N, P] arrays, with bounds on what binary32 evaluation may
add.  u = 2^-24 is half a unit in the last place of binary32, relative; a value that is rounded k times is off by at most k u, to first order, and the
bounds below count the roundings of each term and take the next whole number above, which covers the second order."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -149            # a denormal result is off by half of this
HALF_BF16 = 2.0 ** -8


def factor(norm, max_norm):
    with np.errstate(invalid="ignore"):
        return np.minimum(1.0, max_norm / (np.asarray(norm, dtype=np.float64) + 1e-6))


def rounding(values, bf16):
    """what storing binary32 results in the stack's type may add"""
    return (HALF_BF16 * np.abs(values) + 2.0 ** -134) if bf16 else 0.0


def sgd(p, g, m, lr, momentum, wd, c, nesterov=False, bf16=False):
    """wd: per coordinate; c: per model.  -> new p, new m, bound on p, bound on m"""
    p, g, m = (np.asarray(a, dtype=np.float64) for a in (p, g, m))
    c = np.asarray(c, dtype=np.float64)[:, None]
    d = c * g + wd * p
    new_m = momentum * m + d
    u = d if momentum == 0 else d + momentum * new_m if nesterov else new_m
    size_d = np.abs(c * g) + np.abs(wd * p)          # c and the product: 2; wd's constant, its multiplier, their product, the product with p: 4; the sum: 1
    size_m = momentum * np.abs(m) + size_d           # momentum's constant and the product: 2; d: 5; the sum: 1
    bound_m = 7 * U * size_m + 4 * TINY
    size_u = size_m * (1 + momentum) if nesterov else size_m    # Nesterov: momentum, product, sum: 3 more
    new_p = p - lr * u
    bound_p = U * np.abs(new_p) + lr * 13 * U * size_u + 8 * TINY   # lr's constant, the product, the difference
    return new_p, new_m, bound_p + rounding(np.abs(new_p) + bound_p, bf16), bound_m


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, wd, c, bf16=False):
    """-> new p, m, v and their bounds"""
    p, g, m, v = (np.asarray(a, dtype=np.float64) for a in (p, g, m, v))
    c = np.asarray(c, dtype=np.float64)[:, None]
    t = step + 1
    g = c * g                                        # 2 roundings
    new_m = beta1 * m + (1 - beta1) * g
    new_v = beta2 * v + (1 - beta2) * g * g
    size_m = beta1 * np.abs(m) + (1 - beta1) * np.abs(g)
    bound_m = 6 * U * size_m + 4 * TINY              # g 2, constant, product, sum
    bound_v = 9 * U * new_v + 4 * TINY               # g twice 2, constant, two products, sum: 8; no cancellation
    s1 = 1.0 / (1.0 - beta1 ** t) if beta1 else 1.0
    s2 = 1.0 / np.sqrt(1.0 - beta2 ** t) if beta2 else 1.0
    root = np.sqrt(new_v)
    denom = s2 * root + eps
    ratio = s1 * new_m / denom
    # the root of v: half of v's 9 plus its own and, for denormal v, the root of its absolute error; scale 1, product 1, eps 1, sum 1: 10;  s1 1, product 1, quotient 1
    bound_denom = 10 * U * denom + s2 * np.where(new_v < 1e-30, np.sqrt(4 * TINY), 0.0)
    bound_ratio = s1 * bound_m / denom + np.abs(ratio) * (4 * U + 2 * bound_denom / denom)
    pull = wd * p
    new_p = p - lr * (ratio + pull)
    bound_p = U * np.abs(new_p) + lr * (bound_ratio + 8 * U * (np.abs(ratio) + np.abs(pull))) + 8 * TINY
    return new_p, new_m, new_v, bound_p + rounding(np.abs(new_p) + bound_p, bf16), bound_m, bound_v
