"""The example that runs the operators of rollouts and training together: what was sampled over the paged cache is what the packed attention and the loss
stage score, and the gradients of a whole step are those of the loss in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -8                                                # rounding of bf16


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rollout_step.py")
    spec = importlib.util.spec_from_file_location("rollout_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _step(example, heads, lengths, group, max_new, vocab=768, hidden=256, **kw):
    policy = example.Policy(vocab, hidden, *heads, seed=4)
    stage, loss_stage = example.RolloutStage(), example.LossStage()
    host = torch.Generator().manual_seed(5)
    prompts = [torch.randint(1, vocab, (n,), generator=host).to(torch.int32) for n in lengths]
    batch = example.rollouts(policy, stage, prompts, group, max_new, generator=torch.Generator(device=stage.device).manual_seed(6), **kw)
    rewards = torch.stack([(r < vocab // 2).float().mean() for r in batch["ids"]])
    res = example.loss_and_gradients(policy, stage, loss_stage, batch, rewards, len(lengths), seed=7)
    torch.cuda.synchronize()
    return policy, batch, res


SHAPES = [((8, 2, 64), [1, 17, 40], 4, 24), ((4, 4, 128), [16, 5], 3, 33), ((28, 4, 128), [70], 6, 9)]


@pytest.mark.parametrize("heads,lengths,group,max_new", SHAPES)
def test_sampled_tokens_are_scored_alike(example, heads, lengths, group, max_new):
    """Both sides round q, k, v, the attention's result and h to bf16, the sampled side its logits as well: log-probs differ by a logit's rounding and the
    log-sum's, U max|z| each at most, and by what the roundings of h do to two logits, 2 U |h| |w| by Cauchy and Schwarz for each side."""
    policy, batch, res = _step(example, heads, lengths, group, max_new)
    W = policy.weights["W"].float()
    h_norm = 2.0 * policy.weights["E"].float().norm(dim=1).max().item()        # h = x + attended Wo, the second no longer than the first here
    limit = 2 * U * h_norm * W.norm(dim=1).max().item() * 2
    gap = (res["logp"] - res["old_logp"]).abs()
    assert gap.max().item() <= limit and gap.mean().item() <= limit / 16, (gap.max().item(), gap.mean().item(), limit)
    assert np.isfinite(res["loss"].item()) and res["kept"]["n_kept"] > 0


@pytest.mark.parametrize("heads,lengths,group,max_new", SHAPES[:2])
def test_gradients_of_a_step(example, heads, lengths, group, max_new):
    """Every weight's gradient against the whole step in 64 bits.  Some ten roundings to bf16 in a row, 2-norm U / sqrt(3) each: 7e-3; 2e-2 is the bound."""
    policy, batch, res = _step(example, heads, lengths, group, max_new)
    hq, hkv, D = heads
    w = {n: t.double().cpu().requires_grad_() for n, t in policy.weights.items()}
    kept = res["kept"]
    cut = kept["cut_len"].cpu()
    weight = kept["kept_w"][:kept["n_kept"]].double().cpu()
    adv, old = res["adv"].double().cpu(), res["old_logp"].double().cpu()
    loss, at = 0.0, 0
    for b, full in enumerate(batch["full"]):
        p, L = int(batch["prompt_len"][b]), int(cut[b])
        ids = full[:p + L].long().cpu()
        x = w["E"][ids]
        n = p + L
        q = (x @ w["Wq"]).view(n, hkv, hq // hkv, D)
        k, v = ((x @ w[name]).view(n, hkv, D) for name in ("Wk", "Wv"))
        s = torch.einsum("ihgd,jhd->hgij", q, k) * D ** -0.5
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf"))
        out = torch.einsum("hgij,jhd->ihgd", s.softmax(-1), v).reshape(n, hq * D)
        h = x + out @ w["Wo"]
        logp = (h @ w["W"].t()).log_softmax(-1)
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


def test_cache_in_8_bits(example):
    """3 mantissa bits in keys and values: every element within 2^-4 of itself.  The scores move by as much at most, the log-probs stay those of a similar
    policy; the loss stage takes what was sampled."""
    _, _, res = _step(example, *SHAPES[0], fp8=True)
    gap = (res["logp"] - res["old_logp"]).abs()
    assert gap.mean().item() <= 2.0 ** -4 and np.isfinite(res["loss"].item())


def test_command_runs(example, capsys):
    example.main(["--prompts", "2", "--group", "2", "--max-new", "5", "--vocab", "512", "--hidden", "128", "--q-heads", "4", "--kv-heads", "2", "--steps", "2"])
    assert capsys.readouterr().out.count("step ") == 2
