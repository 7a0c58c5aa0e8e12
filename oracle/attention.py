"""Attention over packed sequences with grouped heads, its gradients, and attention of one token over a paged cache, in fp64
from the formulas, sequence by sequence and head by head.

With `bounds=True` the results come with limits on the error of a computation that holds products and sums in fp32 and rounds
probabilities P, their gradients dS and the results to bf16 (relative error U = 2^-8 each): see the functions."""
import numpy as np

U = 2.0 ** -8                   # largest relative error of rounding to bf16, 8 significant bits


def _visible(n_q, n_k, causal):
    if not causal:
        return np.ones((n_q, n_k), dtype=bool)
    return np.arange(n_k)[None, :] <= np.arange(n_q)[:, None] + (n_k - n_q)


def probabilities(q, k, scale, visible):
    """P [a, b] and the log-sum-exp [a] of the visible scores; a row that sees nothing has P = 0 and -inf, one that sees a score of NaN has NaN.  Masked places are
    never touched by what q and k hold there."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.where(visible, (q @ k.T) * scale, -np.inf)
    m = s.max(axis=1, initial=-np.inf)
    safe = np.where(np.isneginf(m), 0.0, m)
    e = np.where(visible, np.exp(s - safe[:, None]), 0.0)
    total = e.sum(axis=1)
    with np.errstate(divide="ignore"):
        lse = np.where(total == 0, -np.inf, safe + np.log(total))
    return e / np.where(total == 0, 1.0, total)[:, None], lse, s


def _masked_matmul(p, x, visible):
    """p @ x where p is 0 in masked places whatever x holds there."""
    clean = np.where(np.isfinite(x), x, 0.0)
    out = p @ clean
    bad = ~np.isfinite(x)
    if bad.any():
        for j in np.nonzero(bad.any(axis=1))[0]:
            out[np.ix_(visible[:, j], bad[j])] = np.nan
    return out


def attention(q, k, v, cu_q, cu_k, causal=True, scale=None, dout=None, bounds=False):
    """q, dout [n_q, hq, D], k, v [n_k, hkv, D] -> dict(out, lse [hq, n_q] and, with dout, dq, dk, dv); with bounds also
    e_out, e_lse, e_dq, e_dk, e_dv, limits on the absolute errors, element by element:
      out: the probabilities' rounding, U sum_j P_j |v_j|, and the result's, U |out|;
      dv:  the same with dout;
      dq:  scale sum_j |k_j| U (|dS_j| + P_j |dout| . |out|): dS's rounding, and that of the stored `out` inside dout . out;
      dk:  the same, summed over the rows.
    fp32 sums and exponents: a relative error of R = 1e-5 (1 + max |S|) of P (D + 8 roundings of 2^-24 in a score of that size, and
    the exponent's), and of 1e-5 of the terms of dS."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n_q, hq, D = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    r = dict(out=np.zeros_like(q), lse=np.full((hq, n_q), -np.inf))
    if bounds:
        r.update(e_out=np.zeros_like(q), e_lse=np.zeros((hq, n_q)))
    if dout is not None:
        dout = np.asarray(dout, np.float64)
        r.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v))
        if bounds:
            r.update(e_dq=np.zeros_like(q), e_dk=np.zeros_like(k), e_dv=np.zeros_like(v))
    for b in range(len(cu_q) - 1):
        i, j = slice(int(cu_q[b]), int(cu_q[b + 1])), slice(int(cu_k[b]), int(cu_k[b + 1]))
        vis = _visible(i.stop - i.start, j.stop - j.start, causal)
        for h in range(hq):
            g = h // G
            P, lse, S = probabilities(q[i, h], k[j, g], scale, vis)
            out = _masked_matmul(P, v[j, g], vis)
            r["out"][i, h], r["lse"][h, i] = out, lse
            if bounds:
                R = 1e-5 * (1 + np.abs(np.where(vis & np.isfinite(S), S, 0.0)).max(initial=0.0))
                r["e_out"][i, h] = (U + R) * (P @ np.abs(v[j, g])) * 1.02 + U * np.abs(out) * 1.01
                r["e_lse"][h, i] = R
            if dout is None:
                continue
            do = dout[i, h]
            with np.errstate(invalid="ignore"):
                dP = np.where(vis, do @ v[j, g].T, 0.0)
            delta = (do * out).sum(axis=1, keepdims=True)
            dS = np.where(vis, P * (dP - delta), 0.0)
            r["dq"][i, h] = scale * _masked_matmul(dS, k[j, g], vis)
            r["dk"][j, g] += scale * _masked_matmul(dS.T, q[i, h], vis.T)
            r["dv"][j, g] += _masked_matmul(P.T, do, vis.T)
            if bounds:
                e_delta = U * (np.abs(do) * np.abs(out)).sum(axis=1, keepdims=True)
                terms = (np.abs(do) @ np.abs(v[j, g]).T + np.abs(do * out).sum(axis=1, keepdims=True))
                e_dS = U * np.abs(dS) + P * e_delta + R * P * (np.abs(dP) + np.abs(delta)) + 1e-5 * P * terms
                r["e_dq"][i, h] = scale * e_dS @ np.abs(k[j, g]) * 1.02 + U * np.abs(r["dq"][i, h]) * 1.01
                r["e_dk"][j, g] += scale * e_dS.T @ np.abs(q[i, h]) * 1.02
                r["e_dv"][j, g] += (U + R) * (P.T @ np.abs(do)) * 1.02
    if bounds and dout is not None:
        r["e_dk"] += U * np.abs(r["dk"]) * 1.01
        r["e_dv"] += U * np.abs(r["dv"]) * 1.01
    return r


def decode(q, k_cache, v_cache, block_table, seq_lens, scale=None, bounds=False):
    """q [S, hq, D]; caches [pages, hkv, page, D] (values, not codes); tokens with a page outside the cache do not count."""
    q = np.asarray(q, np.float64)
    S, hq, D = q.shape
    n_pages, hkv, page, _ = k_cache.shape
    r = dict(out=np.zeros_like(q), lse=np.full((S, hq), -np.inf))
    if bounds:
        r.update(e_out=np.zeros_like(q), e_lse=np.zeros((S, hq)))
    for b in range(S):
        t = np.arange(min(max(int(seq_lens[b]), 0), block_table.shape[1] * page))
        pages = np.asarray(block_table)[b, t // page]
        t = t[(pages >= 0) & (pages < n_pages)]
        pages = np.asarray(block_table)[b, t // page]
        k, v = (np.asarray(c[pages, :, t % page], np.float64) for c in (k_cache, v_cache))
        one = attention(np.asarray(q[b:b + 1]), k, v, [0, 1], [0, len(t)], causal=False, scale=scale, bounds=bounds)
        for name in r:
            r[name][b] = one[name][0] if name.endswith("out") else one[name][:, 0]
    return r
