"""nat_attn_fwd / nat_attn_bwd against the fp64 oracle: every element within the limits that rounding P, dS and the results to
bf16 allow (oracle/attention.py derives them), and each tensor's error in the 2-norm within 4e-3: a rounding's relative errors of up to
2^-8, evenly spread, have a root mean square of 2^-8 / sqrt(3) = 2.26e-3, two independent ones 3.2e-3."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import attention as oattn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def make(seed, lens_q, lens_k, hq, hkv, D, fused=False, pad=0, spread=1.0):
    """Device tensors q, k, v, dout and offsets; fused: q, k, v are parts of one array (lens_q == lens_k); pad: elements between rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    new = lambda n, h: torch.randn((n, h * D + pad), generator=g, device=DEV, dtype=torch.bfloat16) * spread
    n_q, n_k = sum(lens_q), sum(lens_k)
    cut = lambda x, at, h: x[:, at:at + h * D].unflatten(1, (h, D))
    if fused:
        assert lens_q == lens_k
        x = new(n_q, hq + 2 * hkv)
        q, k, v = cut(x, 0, hq), cut(x, hq * D, hkv), cut(x, (hq + hkv) * D, hkv)
    else:
        q, k, v = cut(new(n_q, hq), 0, hq), cut(new(n_k, hkv), 0, hkv), cut(new(n_k, hkv), 0, hkv)
    cu = lambda l: torch.tensor(np.cumsum([0] + l), dtype=torch.int32, device=DEV)
    return dict(q=q, k=k, v=v, dout=cut(new(n_q, hq), 0, hq), cu_q=cu(lens_q), cu_k=cu(lens_k))


def run(stage, c, causal=True, scale=None, backward=True):
    out, lse = stage.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], causal, scale)
    r = dict(out=out, lse=lse)
    if backward:
        r["dq"], r["dk"], r["dv"] = stage.attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, c["cu_q"], c["cu_k"], causal, scale)
    torch.cuda.synchronize()
    return r


def host(x):
    return x.detach().double().cpu().numpy()


def check(c, r, causal=True, scale=None, names=("out", "lse", "dq", "dk", "dv")):
    ref = oattn.attention(host(c["q"]), host(c["k"]), host(c["v"]), host(c["cu_q"]), host(c["cu_k"]), causal, scale, host(c["dout"]), bounds=True)
    for n in names:
        got, want = host(r[n]), ref[n]
        assert got.shape == want.shape, n
        assert np.array_equal(np.isneginf(got), np.isneginf(want)), n
        fine = np.isfinite(want)
        assert np.isfinite(got[fine]).all(), n
        over = np.abs(np.where(fine, got, 0.0) - np.where(fine, want, 0.0)) - ref["e_" + n] - 1e-30
        assert over.max(initial=-1.0) <= 0, (n, float(over.max()), np.unravel_index(over.argmax(), over.shape))
        norm = np.linalg.norm(want[fine])
        if n != "lse" and norm > 0:
            rel = np.linalg.norm((got - want)[fine]) / norm
            # results that are themselves differences of nearly equal terms (few keys, dS near 0) carry the limits' error, not their own size's
            assert rel <= 4e-3 + np.linalg.norm(ref["e_" + n][fine]) / norm / 4, (n, rel)
    return ref


HEADS = [(4, 4, 64), (8, 2, 64), (7, 1, 64), (2, 2, 128), (8, 2, 128), (14, 2, 128), (16, 1, 128)]
LENS = [
    ([1], [1]), ([2, 1, 3], [2, 1, 3]), ([31, 32, 33], [31, 32, 33]), ([127, 128, 129, 5], [127, 128, 129, 5]),
    ([300, 0, 65, 1], [300, 0, 65, 1]),                       # a sequence without rows
    ([1, 17, 64], [200, 333, 64]),                            # queries behind a cached prefix
    ([70, 130], [20, 0]),                                     # more queries than keys: rows that see nothing, a sequence without keys
]


@pytest.mark.parametrize("hq,hkv,D", HEADS)
@pytest.mark.parametrize("lens", LENS, ids=lambda l: "-".join(map(str, l[0])))
def test_causal(stage, hq, hkv, D, lens):
    c = make(hash((hq, D, len(lens[0]))) % 1000, *lens, hq, hkv, D)
    check(c, run(stage, c))


@pytest.mark.parametrize("lens", LENS[1:], ids=lambda l: "-".join(map(str, l[0])))
@pytest.mark.parametrize("hq,hkv,D", [(6, 2, 64), (6, 2, 128)])
def test_full(stage, hq, hkv, D, lens):
    c = make(3, *lens, hq, hkv, D)
    check(c, run(stage, c, causal=False), causal=False)


@pytest.mark.parametrize("scale,spread", [(0.02, 1.0), (1.0, 1.0), (0.25, 4.0)])
def test_scales_and_peaked_rows(stage, scale, spread):
    c = make(4, [190, 77], [190, 77], 4, 2, 128, spread=spread)
    c["v"] = torch.randn_like(c["v"])
    c["dout"] = torch.randn_like(c["dout"])
    check(c, run(stage, c, scale=scale), scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_parts_of_one_array_and_row_padding(stage, D):
    lens = [90, 1, 150]
    for fused, pad in ((True, 0), (True, 8), (False, 24)):
        c = make(5, lens, lens, 6, 2, D, fused, pad)
        r = run(stage, c)
        ref = run(stage, {n: x.contiguous() for n, x in c.items()})
        for n in r:
            assert torch.equal(r[n], ref[n]), (n, fused, pad)


def test_gradients_into_parts_of_one_array(stage):
    import paper_2603_06619_amd as nat
    hq, hkv, D, n = 6, 2, 64, 200
    c = make(6, [120, 80], [120, 80], hq, hkv, D)
    r = run(stage, c)
    whole = torch.full((n, (hq + 2 * hkv) * D + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    part = lambda at, h: whole[:, at * D:(at + h) * D].unflatten(1, (h, D))
    dq, dk, dv = part(0, hq), part(hq, hkv), part(hq + hkv, hkv)
    ws = torch.empty(nat.attn_bwd_workspace_bytes(n, hq), dtype=torch.uint8, device=DEV)
    nat.nat_attn_bwd(c["q"], c["k"], c["v"], r["out"], r["lse"], c["dout"], c["cu_q"], c["cu_k"], True, D ** -0.5, dq, dk, dv, ws)
    assert torch.equal(dq, r["dq"]) and torch.equal(dk, r["dk"]) and torch.equal(dv, r["dv"])
    assert bool((whole[:, (hq + 2 * hkv) * D:] == 7.0).all())


def test_many_sequences_of_one_to_a_few_rows(stage):
    lens = [1 + i % 3 for i in range(700)]
    c = make(7, lens, lens, 4, 2, 64)
    check(c, run(stage, c))


def test_rows_of_no_sequence_are_left_alone(stage):
    """Offsets that start behind row 0 and end before the last one."""
    import paper_2603_06619_amd as nat
    c = make(8, [60, 40], [60, 40], 2, 2, 64)
    c["cu_q"] = c["cu_k"] = torch.tensor([10, 55, 90], dtype=torch.int32, device=DEV)
    mk = lambda x: torch.full_like(x, 9.0)
    out, lse = mk(c["q"]), torch.full((2, 100), 9.0, device=DEV)
    nat.nat_attn_fwd(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], True, 0.125, out, lse)
    dq, dk, dv = mk(c["q"]), mk(c["k"]), mk(c["v"])
    ws = torch.empty(nat.attn_bwd_workspace_bytes(100, 2), dtype=torch.uint8, device=DEV)
    nat.nat_attn_bwd(c["q"], c["k"], c["v"], out, lse, c["dout"], c["cu_q"], c["cu_k"], True, 0.125, dq, dk, dv, ws)
    for x in (out, dq, dk, dv):
        assert bool((x[:10] == 9).all()) and bool((x[90:] == 9).all())
        assert not bool((x[10:90] == 9).all(-1).any())
    assert bool((lse[:, :10] == 9).all()) and bool((lse[:, 90:] == 9).all())


def test_offsets_beyond_the_arrays_are_clamped(stage):
    c = make(9, [64, 64], [64, 64], 2, 1, 64)
    good = run(stage, c)
    c["cu_q"] = torch.tensor([-5, 64, 4000], dtype=torch.int32, device=DEV)
    c["cu_k"] = torch.tensor([-9, 64, 1 << 30], dtype=torch.int32, device=DEV)
    bad = run(stage, c)
    for n in good:
        assert torch.equal(good[n], bad[n]), n


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_masked_places_hold_has_no_influence(stage, D, value):
    """Keys and values of tokens that come later, and gradients and queries of earlier rows: whatever they hold, rows that do not see
    them (and keys that are not seen by them) keep their results."""
    n, at = 200, 150
    c = make(10, [n, 30], [n, 30], 4, 2, D)
    good = run(stage, c)
    late = {k: x.clone() for k, x in c.items()}
    late["k"][at, :, 1] = value
    late["v"][at, :, D - 3] = value
    r = run(stage, late)
    for name in ("out", "dq"):
        assert torch.equal(r[name][:at], good[name][:at]) and torch.equal(r[name][n:], good[name][n:]), name
        assert not bool(torch.isfinite(r[name][at:n].float()).all()), name
    assert torch.equal(r["lse"][:, :at], good["lse"][:, :at])
    early = {k: x.clone() for k, x in c.items()}
    early["q"][at, :, 5] = value
    early["dout"][at, :, 7] = value
    r = run(stage, early)
    for name in ("dk", "dv"):                  # keys behind row `at` are not seen by it
        assert torch.equal(r[name][at + 1:], good[name][at + 1:]), name
        assert not bool(torch.isfinite(r[name][:at + 1].float()).all()), name
    for name in ("out", "dq"):
        rest = torch.arange(n + 30, device=DEV) != at
        assert torch.equal(r[name][rest], good[name][rest]), name


def test_not_finite_between_sequences(stage):
    """Rows of no sequence may hold anything: last tiles of a sequence reach into them."""
    c = make(11, [100, 100], [100, 100], 2, 2, 128)
    cu = torch.tensor([0, 90, 190], dtype=torch.int32, device=DEV)
    c["cu_q"], c["cu_k"] = cu, cu
    good = run(stage, c)
    for n in ("q", "k", "v", "dout"):
        c[n][190:] = float("nan")
    bad = run(stage, c)
    for n in good:
        a, b = (good[n][:, :190], bad[n][:, :190]) if n == "lse" else (good[n][:190], bad[n][:190])
        assert torch.equal(a, b), n


@pytest.mark.parametrize("hq,hkv,D", [(8, 2, 64), (4, 1, 128)])
def test_gradients_against_differences(stage, hq, hkv, D):
    """Along the gradient itself the oracle's loss sum(out * dout) changes by its length: to 4e-3, as the tensors may differ, and the
    second-order term of the difference."""
    c = make(12, [100, 37], [120, 37], hq, hkv, D)
    r = run(stage, c)
    x = {n: host(c[n]) for n in ("q", "k", "v")}
    f = lambda y: (oattn.attention(y["q"], y["k"], y["v"], host(c["cu_q"]).astype(int), host(c["cu_k"]).astype(int))["out"] * host(c["dout"])).sum()
    for n in ("q", "k", "v"):
        g = host(r["d" + n])
        u = g / np.linalg.norm(g)
        slope = (f({**x, n: x[n] + 1e-4 * u}) - f({**x, n: x[n] - 1e-4 * u})) / 2e-4
        assert abs(slope - np.linalg.norm(g)) <= 4e-3 * np.linalg.norm(g), (n, slope, np.linalg.norm(g))


def test_results_do_not_change_from_run_to_run(stage):
    c = make(13, [500, 333, 64], [500, 333, 64], 8, 2, 128)
    a, b = run(stage, c), run(stage, c)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_another_stream(stage):
    c = make(14, [500, 90], [500, 90], 8, 2, 128)
    ref = run(stage, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = run(stage, c)
    side.synchronize()
    for n in ref:
        assert torch.equal(ref[n], r[n]), n


def test_replays_from_a_graph(stage):
    import paper_2603_06619_amd as nat
    c = make(15, [300, 90], [300, 90], 4, 2, 64)
    ref = run(stage, c)
    o = {n: torch.empty_like(x) for n, x in ref.items()}
    ws = torch.empty(nat.attn_bwd_workspace_bytes(390, 4), dtype=torch.uint8, device=DEV)

    def call():
        nat.nat_attn_fwd(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], True, 0.125, o["out"], o["lse"])
        nat.nat_attn_bwd(c["q"], c["k"], c["v"], o["out"], o["lse"], c["dout"], c["cu_q"], c["cu_k"], True, 0.125, o["dq"], o["dk"], o["dv"], ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rep in range(4):
        for x in o.values():
            x.fill_(3.0)
        ws.fill_(255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for n in ref:
            assert torch.equal(o[n], ref[n]), (rep, n)


def test_rows_beyond_32_bit_offsets(stage):
    """Rows 8192 elements apart, the last sequence more than 2^31 elements into the arrays."""
    n, D = 300000, 64
    base = torch.zeros((n, 8192), dtype=torch.bfloat16, device=DEV)
    small = make(16, [50], [50], 2, 2, D)
    view = lambda at: base[:, at:at + 2 * D].unflatten(1, (2, D))
    c = dict(q=view(0), k=view(1024), v=view(2048), dout=view(4096))
    for name in c:
        c[name][n - 50:] = small[name]
    c["cu_q"] = c["cu_k"] = torch.tensor([n - 50, n], dtype=torch.int32, device=DEV)
    r, ref = run(stage, c), run(stage, small)
    for name in r:
        got = r[name][:, n - 50:] if name == "lse" else r[name][n - 50:]
        assert torch.equal(got, ref[name]), name


def test_long_rows_against_the_oracle_in_places(stage):
    """One sequence of 9001 rows: sampled rows and keys, element by element."""
    n, hq, hkv, D = 9001, 4, 2, 128
    c = make(17, [n], [n], hq, hkv, D)
    r = run(stage, c)
    q, k, v, do = (host(c[x]) for x in ("q", "k", "v", "dout"))
    rows = np.unique(np.concatenate([[0, 1, 63, 64, 127, 128, n - 1], np.random.default_rng(0).integers(0, n, 20)]))
    for h in (0, 3):
        for i in rows:
            P, lse, _ = oattn.probabilities(q[i:i + 1, h], k[:i + 1, h // 2], D ** -0.5, np.ones((1, i + 1), bool))
            out = P @ v[:i + 1, h // 2]
            assert abs(host(r["lse"])[h, i] - lse[0]) <= 1e-4
            assert np.all(np.abs(host(r["out"][i, h]) - out[0]) <= oattn.U * (np.abs(out[0]) + 1.1 * (P @ np.abs(v[:i + 1, h // 2]))[0]))
            dS = P * (do[i, h] @ v[:i + 1, h // 2].T - (do[i, h] * out[0]).sum())
            dq = (dS @ k[:i + 1, h // 2])[0] * D ** -0.5
            terms = (P * (np.abs(do[i, h]) @ np.abs(v[:i + 1, h // 2]).T + np.abs(do[i, h] * out[0]).sum())) @ np.abs(k[:i + 1, h // 2])
            assert np.linalg.norm(host(r["dq"][i, h]) - dq) <= 1.5e-2 * np.linalg.norm(dq) + 1e-5 * D ** -0.5 * np.linalg.norm(terms)
    # a key seen by all rows, and one seen by few, over both heads of its group
    lse = host(r["lse"])
    for j in (0, 4444, n - 70):
        dk, dv = np.zeros(D), np.zeros(D)
        for h in (2, 3):
            s = q[j:, h] @ k[j, 1] * D ** -0.5
            p = np.exp(s - lse[h, j:])
            delta = (do[j:, h] * host(r["out"][j:, h])).sum(-1)
            dv += p @ do[j:, h]
            dk += (p * (do[j:, h] @ v[j, 1] - delta)) @ q[j:, h] * D ** -0.5
        assert np.linalg.norm(host(r["dv"][j, 1]) - dv) <= 1e-2 * np.linalg.norm(dv)
        assert np.linalg.norm(host(r["dk"][j, 1]) - dk) <= 1e-2 * np.linalg.norm(dk)
