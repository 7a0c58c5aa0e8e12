"""nat_attn_bwd where several workgroups share the rows that see a tile of keys (few keys, many rows): within the limits of test_gpu_attention.py, with every
size of workspace."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from test_gpu_attention import check, host, make, run, stage  # noqa: F401 (stage is a fixture)

pytestmark = pytest.mark.gpu


def parts(c, causal=True):
    import paper_2603_06619_amd as nat
    (n_q, hq, D), (n_k, hkv, _) = c["q"].shape, c["k"].shape
    full = nat.attn_bwd_workspace_full_bytes(n_q, n_k, c["cu_q"].numel() - 1, hq, hkv, D, causal)
    return (full - nat.attn_bwd_workspace_bytes(n_q, hq)) // (n_k * hkv * D * 8)


@pytest.mark.parametrize("lens_q,lens_k,hq,hkv,D,causal", [
    ([700], [700], 8, 1, 64, True), ([700], [700], 8, 1, 128, True), ([513], [513], 14, 2, 128, True), ([601], [601], 2, 2, 64, False),
    ([900], [33], 4, 2, 128, False), ([900], [33], 8, 1, 64, True), ([5, 1200, 0, 300], [5, 1200, 0, 300], 6, 2, 64, True), ([300, 900], [1000, 901], 7, 1, 128, True),
    ([129], [129], 60, 1, 128, True),
])
def test_shared_rows(stage, lens_q, lens_k, hq, hkv, D, causal):  # noqa: F811
    c = make(len(lens_q), lens_q, lens_k, hq, hkv, D)
    assert parts(c, causal) > 1
    check(c, run(stage, c, causal=causal), causal=causal)


def test_every_workspace(stage):  # noqa: F811
    """From the least on, the sums are cut as the workspace allows: each result within the limits, dq always the same; what lies behind the workspace and between the
    rows of dk and dv stays."""
    import paper_2603_06619_amd as nat
    hq, hkv, D = 8, 1, 64
    c = make(7, [640, 900], [640, 900], hq, hkv, D)
    n = 1540
    r = run(stage, c)
    slab = n * hkv * D * 8
    least, full = nat.attn_bwd_workspace_bytes(n, hq), nat.attn_bwd_workspace_full_bytes(n, n, 2, hq, hkv, D, True)
    assert (full - least) // slab >= 3
    for size in (least, least + slab, least + 2 * slab, full - slab, full, full + 1000):
        ws = torch.full((size + 4096,), 0xaa, dtype=torch.uint8, device=DEV)
        whole = torch.full((n, 2 * hkv * D + 8), 7.0, dtype=torch.bfloat16, device=DEV)
        dk, dv = (whole[:, at * D:(at + hkv) * D].unflatten(1, (hkv, D)) for at in (0, hkv))
        dq = torch.empty_like(r["dq"])
        nat.nat_attn_bwd(c["q"], c["k"], c["v"], r["out"], r["lse"], c["dout"], c["cu_q"], c["cu_k"], True, D ** -0.5, dq, dk, dv, ws[:size])
        torch.cuda.synchronize()
        assert torch.equal(dq, r["dq"]) and bool((ws[max(size, full):] == 0xaa).all()) and bool((whole[:, 2 * hkv * D:] == 7.0).all())
        check(c, dict(r, dk=dk, dv=dv), names=("dk", "dv"))
        if size >= full:
            assert torch.equal(dk, r["dk"]) and torch.equal(dv, r["dv"])


@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_no_sequence_and_what_is_masked(stage, D):  # noqa: F811
    """Offsets that leave rows out, and infinities and NaN where the mask hides them: later keys and values, and rows outside."""
    import paper_2603_06619_amd as nat
    hq, hkv, n = 8, 1, 1000
    c = make(9, [n], [n], hq, hkv, D)
    c["cu_q"] = c["cu_k"] = torch.tensor([40, 960], dtype=torch.int32, device=DEV)
    assert parts(c) > 1
    inner = {x: c[x][40:960].clone() for x in ("q", "k", "v", "dout")}
    inner["cu_q"] = inner["cu_k"] = torch.tensor([0, 920], dtype=torch.int32, device=DEV)
    ref = run(stage, inner)
    for x in ("q", "k", "v", "dout"):
        c[x][:40] = float("nan")
        c[x][960:] = float("inf")
    out, lse = stage.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"])
    dq, dk, dv = (torch.full_like(c[x], 9.0) for x in ("q", "k", "v"))
    ws = torch.empty(nat.attn_bwd_workspace_full_bytes(n, n, 1, hq, hkv, D, True), dtype=torch.uint8, device=DEV)
    nat.nat_attn_bwd(c["q"], c["k"], c["v"], out, lse, c["dout"], c["cu_q"], c["cu_k"], True, D ** -0.5, dq, dk, dv, ws)
    for got, want in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        assert bool((got[:40] == 9.0).all()) and bool((got[960:] == 9.0).all())
        over = np.abs(host(got[40:960]) - host(ref[want]))
        assert over.max() <= 2.0 ** -7 * np.abs(host(ref[want])).max()         # cut elsewhere: sums of other order, the rounding of the result
    # values that only the last row sees, and that row takes no gradient: the others' gradients stay as they were
    inner["dout"][919] = 0.0
    ref = run(stage, inner)
    inner["k"][919] = inner["v"][919] = 1e30
    r = run(stage, inner)
    assert torch.equal(r["dq"][:919], ref["dq"][:919])


def test_graph(stage):  # noqa: F811
    """Recorded once, replayed on new gradients with eager calls between."""
    c = make(11, [800], [800], 8, 1, 64)
    assert parts(c) > 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(stage, c)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = stage.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"])
            got = stage.attention_backward(c["dout"], c["q"], c["k"], c["v"], out, lse, c["cu_q"], c["cu_k"])
    for i in range(3):
        c["dout"].copy_(torch.randn(c["dout"].shape, device=DEV))
        want = run(stage, c)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        for g, n in zip(got, ("dq", "dk", "dv")):
            assert torch.equal(g, want[n]), (i, n)


def key_parts(c, causal=True):
    import paper_2603_06619_amd as nat
    (n_q, hq, D), (n_k, hkv, _) = c["q"].shape, c["k"].shape
    return nat.attn_fwd_workspace_bytes(n_q, n_k, c["cu_q"].numel() - 1, hq, hkv, D, causal) // (n_q * hq * (D + 2) * 4)


@pytest.mark.parametrize("lens_q,lens_k,hq,hkv,D,causal", [
    ([1], [3001], 4, 4, 64, True), ([16], [8016], 8, 2, 128, True), ([70, 0, 3], [3000, 900, 1700], 7, 1, 128, True), ([5, 200], [4000, 1], 4, 2, 64, True),
    ([700], [2100], 2, 1, 64, True), ([2100], [2100], 2, 1, 64, True), ([2100], [2100], 2, 1, 128, True), ([33], [1100], 60, 1, 64, False), ([65, 64], [4000, 20], 14, 2, 128, False),
])
def test_shared_keys(stage, lens_q, lens_k, hq, hkv, D, causal):  # noqa: F811
    """The forward pass: rows whose keys lie in some parts only, sequences with few keys or none, rows that see nothing."""
    c = make(len(lens_q), lens_q, lens_k, hq, hkv, D)
    assert key_parts(c, causal) > 1
    check(c, run(stage, c, causal=causal, backward=False), causal=causal, names=("out", "lse"))


def test_every_forward_workspace(stage):  # noqa: F811
    import paper_2603_06619_amd as nat
    c = make(3, [40, 9], [4000, 2500], 8, 2, 64)
    c["cu_q"] = torch.tensor([2, 40, 47], dtype=torch.int32, device=DEV)           # rows of no sequence on both sides
    full, part = nat.attn_fwd_workspace_bytes(49, 6500, 2, 8, 2, 64, True), 49 * 8 * 66 * 4
    assert full // part >= 4
    want = None
    for size in (0, part, 2 * part, full, full + 256):
        ws = torch.full((size + 4096,), 0xaa, dtype=torch.uint8, device=DEV)
        out, lse = torch.full_like(c["q"], 9.0), torch.full((8, 49), 9.0, device=DEV)
        nat.nat_attn_fwd(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"], True, 0.125, out, lse, ws[:size])
        torch.cuda.synchronize()
        assert bool((ws[max(size, full):] == 0xaa).all())
        assert bool((out[:2] == 9.0).all()) and bool((out[47:] == 9.0).all()) and bool((lse[:, :2] == 9.0).all()) and bool((lse[:, 47:] == 9.0).all())
        inner = dict(q=c["q"][2:47], k=c["k"], v=c["v"], dout=c["dout"][2:47], cu_q=c["cu_q"] - 2, cu_k=c["cu_k"])
        check(inner, dict(out=out[2:47], lse=lse[:, 2:47]), names=("out", "lse"))
        if size >= full:
            assert want is None or torch.equal(out, want)
            want = out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_what_shared_keys_hold_in_masked_places(stage, D, value):  # noqa: F811
    """Keys and values behind a row's last one, in the same part and in later ones, whatever they hold."""
    c = make(12, [20], [3000], 4, 2, D)
    assert key_parts(c) > 1
    ref = run(stage, c, backward=False)
    c["k"][2990:] = value
    c["v"][2990:] = value
    r = run(stage, c, backward=False)
    assert torch.equal(r["out"][:10], ref["out"][:10]) and torch.equal(r["lse"][:, :10], ref["lse"][:, :10])


def test_forward_graph_and_streams(stage):  # noqa: F811
    """Recorded once and replayed on new queries while the same call runs eagerly on another stream, whose workspace is its own."""
    c = make(13, [24, 7], [5000, 3000], 8, 2, 128)
    assert key_parts(c) > 1
    other = make(14, [24, 7], [5000, 3000], 8, 2, 128)
    want_other = run(stage, other, backward=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(stage, c, backward=False)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = stage.attention(c["q"], c["k"], c["v"], c["cu_q"], c["cu_k"])
    for _ in range(4):
        c["q"].copy_(torch.randn(c["q"].shape, device=DEV))
        want = run(stage, c, backward=False)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        beside = stage.attention(other["q"], other["k"], other["v"], other["cu_q"], other["cu_k"])
        torch.cuda.synchronize()
        assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
        assert torch.equal(beside[0], want_other["out"]) and torch.equal(beside[1], want_other["lse"])
