"""The 2-norm of each tensor's error against what independent roundings give, which is far less than the sum of their largest values: a small missing term, a truncated
P or an inaccurate delta shows here.  And the careful pass of dk, dv where several workgroups share a tile's rows.

A rounding to bf16 has a relative error of root mean square S = 2^-8 / sqrt(3) at most.  With errors independent of one another, element by element,
    out:  S^2 (sum_j (P_j v_j)^2 + out^2)                     (P, and the result);   dv: the same with P^T and dout;
    dq:   scale^2 (S^2 sum_j (dS_j k_j)^2 + var(delta) (sum_j P_j k_j)^2) + S^2 dq^2,   var(delta) = sum_e dout_e^2 var(out_e);
    dk:   scale^2 sum_i (S^2 dS_i^2 + var(delta_i) P_i^2) q_i^2 + S^2 dk^2.
The errors of many elements come close to the root of the summed variances; 1.25 of it is allowed (S is that of the worst mantissa; over all it is 0.72 of it).  For out and dv
of normal inputs that is at most 3.2e-3 of the tensor, and 4e-3 is asked."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle.attention import _visible, probabilities
from test_gpu_attention import host, make, run, stage  # noqa: F401 (stage is a fixture)
from test_gpu_attention_split import key_parts, parts

pytestmark = pytest.mark.gpu
S2 = (2.0 ** -8) ** 2 / 3


def variances(c, causal):
    """The tensors in 64 bits, and the sums of their elements' variances."""
    q, k, v, do = (host(c[x]) for x in ("q", "k", "v", "dout"))
    cu_q, cu_k = host(c["cu_q"]).astype(int), host(c["cu_k"]).astype(int)
    G, scale = q.shape[1] // k.shape[1], q.shape[2] ** -0.5
    r = {n: np.zeros_like(x) for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    var = {n: np.zeros_like(x) for n, x in r.items()}
    for b in range(len(cu_q) - 1):
        i, j = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        vis = _visible(i.stop - i.start, j.stop - j.start, causal)
        for h in range(q.shape[1]):
            g = h // G
            P, _, _ = probabilities(q[i, h], k[j, g], scale, vis)
            out = P @ v[j, g]
            dP = do[i, h] @ v[j, g].T
            dS = P * (dP - (do[i, h] * out).sum(1, keepdims=True))
            r["out"][i, h], r["dq"][i, h] = out, scale * dS @ k[j, g]
            r["dk"][j, g] += scale * dS.T @ q[i, h]
            r["dv"][j, g] += P.T @ do[i, h]
            v_out = S2 * ((P ** 2) @ v[j, g] ** 2 + out ** 2)
            v_delta = (do[i, h] ** 2 * v_out).sum(1, keepdims=True)
            var["out"][i, h] = v_out
            var["dq"][i, h] = scale ** 2 * (S2 * (dS ** 2) @ k[j, g] ** 2 + v_delta * (P @ k[j, g]) ** 2) + S2 * r["dq"][i, h] ** 2
            var["dk"][j, g] += scale ** 2 * (S2 * dS ** 2 + v_delta * P ** 2).T @ q[i, h] ** 2
            var["dv"][j, g] += S2 * (P ** 2).T @ do[i, h] ** 2
    for n in ("dk", "dv"):
        var[n] += S2 * r[n] ** 2
    return r, {n: x.sum() for n, x in var.items()}


CASES = [([300, 0, 65, 1], [300, 0, 65, 1], 14, 2, 128, True), ([300, 0, 65, 1], [300, 0, 65, 1], 14, 2, 64, True), ([700], [700], 8, 1, 128, True),
         ([700], [700], 8, 1, 64, True), ([120, 250], [500, 260], 8, 2, 128, True), ([400, 90], [300, 90], 4, 4, 64, True), ([300, 128], [200, 400], 6, 2, 128, False),
         ([1500], [1500], 4, 1, 64, True), ([200], [3000], 4, 2, 128, True), ([1000], [60], 8, 2, 128, False)]


@pytest.mark.parametrize("lens_q,lens_k,hq,hkv,D,causal", CASES)
def test_errors_are_those_of_independent_roundings(stage, lens_q, lens_k, hq, hkv, D, causal):  # noqa: F811
    c = make(51, lens_q, lens_k, hq, hkv, D)
    got = run(stage, c, causal=causal)
    want, var = variances(c, causal)
    for n in ("out", "dq", "dk", "dv"):
        err, norm = np.linalg.norm(host(got[n]) - want[n]), np.linalg.norm(want[n])
        assert err <= 1.25 * np.sqrt(var[n]), (n, err / norm, np.sqrt(var[n]) / norm)
        if n in ("out", "dv"):
            assert err <= 4e-3 * norm, (n, err / norm)


def test_cases_reach_the_shared_kernels():
    """Some of the cases above have rows and keys that several workgroups share."""
    cases = [(make(51, *c[:5]), c[5]) for c in CASES]
    assert sum(parts(*c) > 1 for c in cases) >= 3 and sum(key_parts(*c) > 1 for c in cases) >= 1


@pytest.mark.parametrize("hq,hkv,D", [(8, 1, 64), (8, 1, 128), (4, 2, 64), (14, 2, 128)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_masked_rows_among_shared_ones(stage, hq, hkv, D, value):  # noqa: F811
    """Early rows of a long sequence that hold infinities or NaN: keys behind them keep their gradients bit for bit, in the tile of the mask's edge and in later ones; keys
    that they see do not hide them."""
    n = 1000
    c = make(52, [n], [n], hq, hkv, D)
    assert parts(c) > 1
    good = run(stage, c)
    for at in (5, 130, 470, 998):
        bad = {x: t.clone() for x, t in c.items()}
        bad["q"][at, :, 5] = value
        bad["dout"][at, :, 7] = value
        r = run(stage, bad)
        for name in ("dk", "dv"):
            assert torch.equal(r[name][at + 1:], good[name][at + 1:]), (name, at)
            assert not bool(torch.isfinite(r[name][:at + 1].float()).all(-1).any()), (name, at)
        rest = torch.arange(n, device=DEV) != at
        for name in ("out", "dq"):
            assert torch.equal(r[name][rest], good[name][rest]), (name, at)
