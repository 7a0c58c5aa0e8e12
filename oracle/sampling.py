"""Sampling from its definition, one row at a time, with Python's whole numbers."""
import math

import numpy as np

ONE = 1 << 40


def weights(z, temperature):
    """Whole-number weights of float32 logits (see `sample`)."""
    z = np.asarray(z, np.float32)
    z = np.where(np.isnan(z), np.float32(-np.inf), z)
    top = z.max()
    if top == -np.inf:
        return [0] * len(z), z
    if not temperature > 0:
        first = int(np.argmax(z))
        return [ONE if i == first else 0 for i in range(len(z))], z
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(z == top, np.float32(0), z - top)
        y = np.where(x == 0, np.float32(0), x * (np.float32(1.4426950408889634) / np.float32(temperature)))
    a = np.where(z == -np.inf, 0.0, np.rint(np.exp2(y.astype(np.float64)) * ONE))
    return [int(w) for w in a], z


def filtered(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weights after the filters."""
    a, z = weights(z, temperature)
    order = sorted(range(len(z)), key=lambda i: (-float(z[i]), i))
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1.0:
        total = sum(a[i] for i in order)
        reach = max(1, (int(max(top_p, 0.0) * 2 ** 32) * total) >> 32)
        kept, run = [], 0
        for i in order:
            if run >= reach:
                break
            kept.append(i)
            run += a[i]
        order = kept
    least = math.ceil(min(min_p, 1.0) * ONE) if min_p > 0 else 0
    keep = set(i for i in order if a[i] >= least)
    return [a[i] if i in keep else 0 for i in range(len(z))], z


def sample(z, word, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log soft-max of the logits at it, log of the probability it was drawn with); (-1, nan, nan) without a logit above -inf."""
    a, z = filtered(z, temperature, top_k, top_p, min_p)
    total = sum(a)
    if total == 0:
        return -1, math.nan, math.nan
    target, run = (int(word) * total) >> 32, 0
    for i, w in enumerate(a):
        run += w
        if run > target:
            break
    z64 = z.astype(np.float64)
    top = z64.max()
    if np.isposinf(top):
        logp = -math.log(int(np.isposinf(z64).sum()))
    else:
        logp = float(z64[i] - top - math.log(np.exp(z64 - top).sum()))
    return i, logp, math.log(a[i] / total)
