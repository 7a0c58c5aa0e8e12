"""The example's step with everything between token ids and attention in use: queries and keys normed and rotated, the cache in 4 bits, pages from the stack and back, tied weights.
What was sampled over the paged cache is what the packed attention and the loss stage score, and the gradients of a whole step are those of the loss in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_rollout_step import U, example  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
SHAPES = [((8, 2, 64), [1, 17, 40], 4, 24), ((4, 4, 128), [16, 5], 3, 33)]


def step(example, heads, lengths, group, max_new, tied=False, vocab=768, hidden=256, **kw):  # noqa: F811
    policy = example.Policy(vocab, hidden, *heads, seed=4, rotate=True, tied=tied)
    stage, loss_stage = example.RolloutStage(), example.LossStage()
    host = torch.Generator().manual_seed(5)
    prompts = [torch.randint(1, vocab, (n,), generator=host).to(torch.int32) for n in lengths]
    batch = example.rollouts(policy, stage, prompts, group, max_new, generator=torch.Generator(device=stage.device).manual_seed(6), **kw)
    rewards = torch.stack([(r < vocab // 2).float().mean() for r in batch["ids"]])
    res = example.loss_and_gradients(policy, stage, loss_stage, batch, rewards, len(lengths), seed=7)
    torch.cuda.synchronize()
    return policy, batch, res


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("heads,lengths,group,max_new", SHAPES)
def test_sampled_tokens_are_scored_alike(example, heads, lengths, group, max_new, tied):  # noqa: F811
    """Both sides round q, k, v (queries and keys twice), the attention's result and h to bf16, the sampled side its logits as well: log-probs differ by a logit's rounding and the
    log-sum's, U max|z| each at most, and by what the roundings of h do to two logits, 2 U |h| |w| by Cauchy and Schwarz for each side."""
    policy, batch, res = step(example, heads, lengths, group, max_new, tied)
    W = policy.head.float()
    h_norm = 2.0 * policy.scale * policy.weights["E"].float().norm(dim=1).max().item()        # h = x + attended Wo, the second no longer than the first here
    limit = 2 * U * h_norm * W.norm(dim=1).max().item() * 2
    gap = (res["logp"] - res["old_logp"]).abs()
    assert gap.max().item() <= limit and gap.mean().item() <= limit / 16, (gap.max().item(), gap.mean().item(), limit)
    assert np.isfinite(res["loss"].item()) and res["kept"]["n_kept"] > 0
    pages = len(lengths) * group * -(-(max(lengths) + max_new) // 16)
    assert batch["free_pages"].tolist() == [pages, 0]                                        # all of them are back


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("heads,lengths,group,max_new", SHAPES)
def test_gradients_of_a_step(example, heads, lengths, group, max_new, tied):  # noqa: F811
    """Every weight's gradient against the whole step in 64 bits.  Some twelve roundings to bf16 in a row, 2-norm U / sqrt(3) each: 8e-3; 2e-2 is the bound."""
    policy, batch, res = step(example, heads, lengths, group, max_new, tied)
    hq, hkv, D = heads
    w = {n: t.double().cpu().requires_grad_() for n, t in policy.weights.items()}
    head = w["E" if tied else "W"]
    assert set(res["grads"]) == set(w)
    kept = res["kept"]
    cut = kept["cut_len"].cpu()
    weight = kept["kept_w"][:kept["n_kept"]].double().cpu()
    adv, old = res["adv"].double().cpu(), res["old_logp"].double().cpu()
    freq = policy.inv_freq.cpu()

    def turned(x, norm):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * norm
        angle = torch.arange(x.shape[0], dtype=torch.float64)[:, None, None] * freq
        a, b = x.chunk(2, -1)
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)
    loss, at = 0.0, 0
    for b, full in enumerate(batch["full"]):
        p, L = int(batch["prompt_len"][b]), int(cut[b])
        ids = full[:p + L].long().cpu()
        n = p + L
        x = w["E"][ids] * policy.scale
        q, k = turned((x @ w["Wq"]).view(n, hq, D), w["Nq"]), turned((x @ w["Wk"]).view(n, hkv, D), w["Nk"])
        v = (x @ w["Wv"]).view(n, hkv, D)
        s = torch.einsum("ihgd,jhd->hgij", q.view(n, hkv, hq // hkv, D), k) * D ** -0.5
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf"))
        out = torch.einsum("hgij,jhd->ihgd", s.softmax(-1), v).reshape(n, hq * D)
        h = x + out @ w["Wo"]
        logp = (h @ head.t()).log_softmax(-1)
        for t in range(L):
            ratio = (logp[p + t - 1, ids[p + t]] - old[at]).exp()
            loss = loss - weight[at] * torch.minimum(ratio * adv[b], ratio.clamp(0.8, 1.2) * adv[b])
            at += 1
    assert at == kept["n_kept"]
    loss.backward()
    for name, t in w.items():
        err = (res["grads"][name].double().cpu() - t.grad).norm() / t.grad.norm()
        assert err.item() <= 2e-2, (name, err.item())
    assert abs(res["loss"].item() - loss.item()) <= 2e-2 * (weight * adv[kept["kept_seq"][:at].long().cpu()].abs()).sum().item()


def test_cache_in_4_bits(example):  # noqa: F811
    """1 mantissa bit in keys and values: every element within a quarter of itself.  The log-probs stay those of a similar policy; the loss stage takes what was sampled."""
    _, batch, res = step(example, *SHAPES[0], fp4=True)
    gap = (res["logp"] - res["old_logp"]).abs()
    assert gap.mean().item() <= 2.0 ** -2 and np.isfinite(res["loss"].item())


def test_command_runs(example, capsys):  # noqa: F811
    common = ["--prompts", "2", "--group", "2", "--max-new", "5", "--vocab", "512", "--hidden", "128", "--q-heads", "4", "--kv-heads", "2", "--steps", "2"]
    example.main(common + ["--rotate", "--fp4"])
    example.main(common + ["--rotate", "--tied"])
    assert capsys.readouterr().out.count("step ") == 4
