"""nat_qk_norm_rope and its backward pass against the formulas in 64 bits, element by element within the limits that oracle/heads.py derives."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import heads as ohead

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def case(seed, n, hq, hkv, D, R, dtype, norms=(True, True), most=40000, theta=1e6, size=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=g, device=DEV)
    rows = lambda h: (size * new(n, h, D) * torch.exp(new(n, h, 1))).to(dtype)
    weight = lambda on: (1 + 0.3 * new(D)).to(dtype) if on else None
    c = dict(q=rows(hq), k=rows(hkv), q_weight=weight(norms[0]), k_weight=weight(norms[1]), position_ids=None, inv_freq=None)
    if R:
        c["position_ids"] = torch.randint(most, (n,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        c["inv_freq"] = theta ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device=DEV) / R)
    return c, (new(n, hq, D).to(dtype), new(n, hkv, D).to(dtype))


def host(t):
    return None if t is None else t.double().cpu().numpy()


def reference(c, name, **kw):
    return ohead.norm_rotate(host(c[name]), host(c[name + "_weight"]), host(c["position_ids"]), host(c["inv_freq"]), half=HALF[c[name].dtype], **kw)


def close(got, want, limit):
    got = host(got)
    assert got.shape == want.shape and np.all(np.abs(got - want) <= limit + 1e-37), float((np.abs(got - want) / (limit + 1e-37)).max())


def check(c, got, **kw):
    for name, y in zip("qk", got):
        close(y, *reference(c, name, **kw))


def check_backward(c, grads, got, **kw):
    for name, dout, dx, dw in zip("qk", grads, got[:2], got[2:]):
        n, heads = c[name].shape[:2]
        # a lane: a row of 3072 rows at a time, 8 heads of these; then 4 steps across lanes, 4 wavefronts, 768 workgroups by 32 walkers and their sum
        chain = -(-n // 3072) * -(-heads // 8) + 4 + 4 + 24 + 32
        ref = ohead.norm_rotate_backward(host(dout), host(c[name]), host(c[name + "_weight"]), host(c["position_ids"]), host(c["inv_freq"]),
                                         half=HALF[dout.dtype], chain=chain, **kw)
        close(dx, ref["dx"], ref["e_dx"])
        assert (dw is None) == (c[name + "_weight"] is None)
        if dw is not None:
            assert dw.dtype == torch.float32
            close(dw, ref["dw"], ref["e_dw"])


SHAPES = [(1, 1, 1, 64, 64), (2, 8, 2, 128, 128), (5, 3, 7, 64, 32), (33, 28, 4, 128, 128), (64, 32, 8, 128, 64), (7, 16, 16, 64, 16), (3, 9, 1, 128, 112),
          (257, 5, 5, 64, 48), (2, 1, 65, 128, 16), (19, 12, 1, 128, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,hq,hkv,D,R", SHAPES)
def test_forward_and_backward(stage, dtype, interleaved, n, hq, hkv, D, R):
    c, grads = case(n + D, n, hq, hkv, D, R, dtype)
    kw = dict(eps=1e-6, interleaved=interleaved)
    check(c, stage.norm_rotate(**c, **kw), **kw)
    check_backward(c, grads, stage.norm_rotate_backward(*grads, **c, **kw), **kw)


@pytest.mark.parametrize("norms", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("D,R", [(64, 64), (128, 96)])
def test_weights_on_one_side_or_none(stage, norms, D, R):
    c, grads = case(3, 41, 6, 2, D, R, torch.bfloat16, norms)
    check(c, stage.norm_rotate(**c, eps=1e-5), eps=1e-5)
    check_backward(c, grads, stage.norm_rotate_backward(*grads, **c, eps=1e-5), eps=1e-5)


def test_neither_norm_nor_rotation_copies(stage):
    c, grads = case(4, 9, 3, 2, 64, 0, torch.bfloat16, (False, False))
    q, k = stage.norm_rotate(**c)
    assert torch.equal(q, c["q"]) and torch.equal(k, c["k"])
    dq, dk, a, b = stage.norm_rotate_backward(*grads, **c)
    assert torch.equal(dq, grads[0]) and torch.equal(dk, grads[1]) and a is None and b is None


@pytest.mark.parametrize("positions", [[0, 1, 2, 3], [2 ** 31 - 1, 2 ** 30 + 7, 123456789, 1000003], [-5, -1, -2 ** 31, -77]])
def test_far_and_negative_positions(stage, positions):
    c, grads = case(5, 4, 2, 2, 128, 128, torch.float32, theta=1e4)
    c["position_ids"] = torch.tensor(positions, dtype=torch.int32, device=DEV)
    check(c, stage.norm_rotate(**c))
    check_backward(c, grads, stage.norm_rotate_backward(*grads, **c))


@pytest.mark.parametrize("size", [1e-30, 1e-4, 1e10, 3e19, 1e36])
def test_sizes_whose_squares_leave_the_range(stage, size):
    c, grads = case(6, 12, 4, 2, 64, 64, torch.float32, size=size)
    c["q"], c["k"] = (x.clamp(-3e38, 3e38) for x in (c["q"], c["k"]))
    check(c, stage.norm_rotate(**c))
    check_backward(c, grads, stage.norm_rotate_backward(*grads, **c))


def test_rows_of_zeros_and_not_finite(stage):
    c, grads = case(7, 6, 8, 8, 64, 64, torch.bfloat16)
    c["q"][1], c["q"][2, 3], c["q"][3, 1, 5], c["q"][4, 2, 60] = 0, 0, float("nan"), float("inf")
    q, k = stage.norm_rotate(**c)
    assert bool((q[1] == 0).all()) and bool((q[2, 3] == 0).all()) and bool(q[3, 1].isnan().all())
    assert bool(q[4, 2, [28, 60]].isnan().all()) and bool((q[4, 2, :28] == 0).all())            # inf / inf, and finite / inf
    clean = torch.ones((6, 8), dtype=torch.bool, device=DEV)
    clean[3, 1] = clean[4, 2] = False
    c["q"][~clean] = 0
    again, _ = stage.norm_rotate(**c)
    assert torch.equal(q[clean], again[clean])                                                  # the other heads do not see it
    dq, dk, dqw, dkw = stage.norm_rotate_backward(*grads, **c)
    assert bool(dq.isfinite().all()) and bool(dqw.isfinite().all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_in_place_and_rows_left_alone(stage, dtype):
    import paper_2603_06619_amd as nat
    n, hq, hkv, D = 21, 6, 2, 64
    c, grads = case(8, n, hq, hkv, D, 64, dtype)
    want, back = stage.norm_rotate(**c), stage.norm_rotate_backward(*grads, **c)
    whole = torch.full((n + 2, (hq + 2 * hkv) * D + 8), 7.0, dtype=dtype, device=DEV)                 # queries, keys and values of one projection
    parts = whole[:n, :(hq + 2 * hkv) * D].unflatten(1, (hq + 2 * hkv, D))
    q, k = parts[:, :hq], parts[:, hq:hq + hkv]
    q.copy_(c["q"])
    k.copy_(c["k"])
    args = (c["q_weight"], c["k_weight"], c["position_ids"], c["inv_freq"], 1e-6, False)
    got = stage.norm_rotate(q, k, *args[2:4], *args[:2])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws = torch.empty(nat.qk_norm_rope_bwd_workspace_bytes(n, D), dtype=torch.uint8, device=DEV)
    dw = torch.ones((2, D), device=DEV)
    g = [torch.cat((x, x), 1)[:, :x.shape[1]] for x in grads]                                        # strided, and replaced by what they become
    nat.nat_qk_norm_rope_bwd(q, k, *args, *g, *g, dw[0], dw[1], True, ws)
    assert torch.equal(g[0], back[0]) and torch.equal(g[1], back[1])
    assert torch.equal(dw[0], back[2] + 1) and torch.equal(dw[1], back[3] + 1)
    nat.nat_qk_norm_rope(q, k, *args, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert bool((whole[n:] == 7).all()) and bool((whole[:, (hq + hkv) * D:] == 7).all())


def test_one_row_for_all(stage):
    c, grads = case(9, 30, 4, 2, 128, 128, torch.bfloat16)
    c["q"], dout = c["q"][:1].expand(30, 4, 128), grads[1][:1].expand(30, 2, 128)
    q, k = stage.norm_rotate(**c)
    own = dict(c, q=c["q"].contiguous())
    assert torch.equal(q, stage.norm_rotate(**own)[0])
    for a, b in zip(stage.norm_rotate_backward(grads[0], dout, **c), stage.norm_rotate_backward(grads[0], dout.contiguous(), **own)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n,hq,hkv,D", [(20011, 4, 2, 64), (8193, 9, 3, 128), (3000, 40, 40, 128)])
def test_many_rows_and_runs(stage, n, hq, hkv, D):
    c, grads = case(10, n, hq, hkv, D, D, torch.bfloat16)
    check(c, stage.norm_rotate(**c))
    got = stage.norm_rotate_backward(*grads, **c)
    check_backward(c, grads, got)
    for _ in range(3):
        for a, b in zip(got, stage.norm_rotate_backward(*grads, **c)):
            assert torch.equal(a, b)


def test_no_rows(stage):
    import paper_2603_06619_amd as nat
    c, grads = case(11, 0, 4, 2, 64, 64, torch.bfloat16)
    q, k = stage.norm_rotate(**c)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    dq, dk, dqw, dkw = stage.norm_rotate_backward(*grads, **c)
    assert dq.shape == q.shape and bool((dqw == 0).all()) and bool((dkw == 0).all())
    dqw.fill_(3)
    nat.nat_qk_norm_rope_bwd(c["q"], c["k"], c["q_weight"], c["k_weight"], c["position_ids"], c["inv_freq"], 1e-6, False, *grads, dq, dk, dqw, dkw, True, None)
    assert bool((dqw == 3).all()) and bool((dkw == 0).all())


def test_gradients_against_differences(stage):
    """In fp32 rows with steps of 2^-6: differences are good to h^2 times a third derivative (of order 1 here) and to the rounding of the results over h."""
    c, grads = case(12, 8, 2, 1, 64, 64, torch.float32, size=1.0)
    back = stage.norm_rotate_backward(*grads, **c)
    f = lambda d: sum(float((y.double() * g.double()).sum()) for y, g in zip(stage.norm_rotate(**d), grads))
    gen = torch.Generator(device=DEV).manual_seed(13)
    h = 2.0 ** -6
    for name, grad in (("q", back[0]), ("k", back[1]), ("q_weight", back[2]), ("k_weight", back[3])):
        u = torch.randn(c[name].shape, generator=gen, device=DEV)
        u = u / u.norm()
        want = float((grad.double() * u.double()).sum())
        got = (f(dict(c, **{name: c[name] + h * u})) - f(dict(c, **{name: c[name] - h * u}))) / (2 * h)
        scale = float(grad.double().norm())
        assert abs(got - want) <= 2 * h * h * scale * 4 + 1e-4 * scale, (name, got, want, scale)


@pytest.mark.parametrize("R", [0, 64, 128])
def test_a_backward_pass_of_more_than_the_caches_hold(stage, R):
    """Rows are independent, so halves, which are held, give the same rows; the weights' gradients against sums in 64 bits (R = 0: of dout_i x_i / sqrt(mean x^2 + eps), each term
    off by 6 roundings)."""
    import paper_2603_06619_amd as nat
    n, hq, hkv, D = 4600, 64, 16, 128
    assert n * (hq + hkv) * D * 2 * 3 > 1 << 28 > n // 2 * (hq + hkv) * D * 2 * 3
    c, grads = case(14, n, hq, hkv, D, R, torch.bfloat16)
    dq, dk, dqw, dkw = stage.norm_rotate_backward(*grads, **c)
    for rows in (slice(0, n // 2), slice(n // 2, n)):
        part = dict(c, q=c["q"][rows], k=c["k"][rows], position_ids=c["position_ids"][rows] if R else None)
        a, b, _, _ = stage.norm_rotate_backward(*(x[rows] for x in grads), **part)
        assert torch.equal(a, dq[rows]) and torch.equal(b, dk[rows])
    if R == 0:
        chain = -(-n // 3072) * -(-hq // 8) + 4 + 4 + 24 + 32 + 6
        for x, g, got in ((c["q"], grads[0], dqw), (c["k"], grads[1], dkw)):
            x = x.double()
            terms = g.double() * x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            assert bool(((got.double() - terms.sum((0, 1))).abs() <= chain * 2.0 ** -24 * terms.abs().sum((0, 1))).all())
    ws = torch.empty(nat.qk_norm_rope_bwd_workspace_bytes(n, D), dtype=torch.uint8, device=DEV)
    mine, dw = [g.clone() for g in grads], torch.empty((2, D), device=DEV)
    nat.nat_qk_norm_rope_bwd(c["q"], c["k"], c["q_weight"], c["k_weight"], c["position_ids"], c["inv_freq"], 1e-6, False, *mine, *mine, dw[0], dw[1], False, ws)
    assert torch.equal(mine[0], dq) and torch.equal(mine[1], dk) and torch.equal(dw[0], dqw) and torch.equal(dw[1], dkw)


def test_rows_beyond_32_bit_offsets(stage):
    """Rows 2^30 elements apart, of one array of 4.3 GB."""
    import paper_2603_06619_amd as nat
    n, hq, hkv, D = 3, 6, 2, 128
    c, grads = case(15, n, hq, hkv, D, D, torch.bfloat16)
    want, back = stage.norm_rotate(**c), stage.norm_rotate_backward(*grads, **c)
    whole, at, apart = torch.empty(2 * 2 ** 30 + 8 * (hq + hkv) * D, dtype=torch.bfloat16, device=DEV), 0, []
    for x in (c["q"], c["k"], *grads, *want, *back[:2]):
        apart.append(whole.as_strided(x.shape, (2 ** 30, D, 1), at))
        at += x.shape[1] * D
    for x, y in zip(apart, (c["q"], c["k"], *grads)):
        x.copy_(y)
    q, k, dq_out, dk_out, q_out, k_out, dq, dk = apart
    args = (q, k, c["q_weight"], c["k_weight"], c["position_ids"], c["inv_freq"], 1e-6, False)
    nat.nat_qk_norm_rope(*args, q_out, k_out)
    assert torch.equal(q_out, want[0]) and torch.equal(k_out, want[1])
    ws = torch.empty(nat.qk_norm_rope_bwd_workspace_bytes(n, D), dtype=torch.uint8, device=DEV)
    dw = torch.empty((2, D), device=DEV)
    nat.nat_qk_norm_rope_bwd(*args, dq_out, dk_out, dq, dk, dw[0], dw[1], False, ws)
    assert all(torch.equal(x, y) for x, y in zip((dq, dk, dw[0], dw[1]), back))
