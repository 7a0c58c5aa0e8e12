"""One step of reinforcement learning with a small policy (embedding, one attention layer, head), every operator where it is used:

  rollouts   attention over the packed prompts, their keys and values into a paged cache; then token by token sampling, cache write and attention over
             the cache.  The sampled tokens' log-probabilities are the behaviour log-probs of the loss;
  loss       advantages, random prefix cutting, the truncated batch, attention over it, the loss stage;
  gradients  of the head from the loss stage, of the layer through the attention's backward pass.

Projections are plain torch products.  Run it as `python examples/rollout_step.py` (needs the built library and a GPU)."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_06619_amd as nat                          # noqa: E402
from paper_2603_06619_amd.rollout import PagedCache, RolloutStage  # noqa: E402
from paper_2603_06619_amd.stage import LossStage            # noqa: E402


class Policy:
    """h = x + attention(x Wq, x Wk, x Wv) Wo, x = E[ids]; logits = h W^T."""

    def __init__(self, vocab, hidden, q_heads, kv_heads, head_dim, seed=0, device="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        new = lambda rows, cols, std: (torch.randn(rows, cols, generator=g) * std).to(torch.bfloat16).to(device)
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.weights = dict(E=new(vocab, hidden, 1.0), Wq=new(hidden, q_heads * head_dim, hidden ** -0.5),
                            Wk=new(hidden, kv_heads * head_dim, hidden ** -0.5), Wv=new(hidden, kv_heads * head_dim, hidden ** -0.5),
                            Wo=new(q_heads * head_dim, hidden, (q_heads * head_dim) ** -0.5), W=new(vocab, hidden, hidden ** -0.5))

    def qkv(self, x):
        w, n = self.weights, x.shape[0]
        return ((x @ w["Wq"]).view(n, self.q_heads, self.head_dim), (x @ w["Wk"]).view(n, self.kv_heads, self.head_dim),
                (x @ w["Wv"]).view(n, self.kv_heads, self.head_dim))

    def hidden(self, x, attended):
        return x + attended.reshape(x.shape[0], -1) @ self.weights["Wo"]


def rollouts(policy, stage, prompts, group, max_new, page_size=16, fp8=False, temperature=1.0, top_p=1.0, end_id=0, generator=None):
    """`group` continuations of every prompt (a list of int32 id tensors), of up to max_new tokens, the last of them end_id or not.
    Returns per rollout: ids of prompt and response, response length, behaviour log-probs."""
    dev, E, W = stage.device, policy.weights["E"], policy.weights["W"]
    B = len(prompts) * group
    lens = torch.tensor([len(p) for p in prompts])
    cu = torch.cat((torch.zeros(1, dtype=torch.int64), lens.cumsum(0)))
    x = E[torch.cat(prompts).to(dev).long()]
    q, k, v = policy.qkv(x)
    out, _ = stage.attention(q, k, v, cu.to(torch.int32).to(dev))
    last = cu[1:] - 1
    h = policy.hidden(x, out)[last.to(dev)].repeat_interleave(group, 0)

    # pages of a rollout: any, in any order
    width = (int(lens.max()) + max_new + page_size - 1) // page_size
    cache = PagedCache.empty(B * width, policy.kv_heads, page_size, policy.head_dim, fp8=fp8, device=dev)
    table = torch.randperm(B * width).to(torch.int32).view(B, width)
    slot = lambda b, t: table[b, t // page_size].long() * page_size + t % page_size
    rows = torch.cat([torch.arange(cu[b // group], cu[b // group + 1]) for b in range(B)])
    slots = torch.cat([slot(b, torch.arange(lens[b // group])) for b in range(B)])
    stage.write_cache(cache, k[rows.to(dev)], v[rows.to(dev)], slots.to(dev))

    length = lens.repeat_interleave(group)
    every = torch.arange(B)
    device_table = table.to(dev)
    seq_lens = length.to(torch.int32).to(dev)
    settings = dict(temperature=torch.full((B,), temperature, device=dev), top_p=torch.full((B,), top_p, device=dev))
    ids, logp = [], []
    for t in range(max_new):
        word = torch.randint(-2 ** 31, 2 ** 31, (B,), dtype=torch.int32, device=dev, generator=generator)
        drawn = stage.sample(h @ W.t(), word, **settings)
        ids.append(drawn["ids"])
        logp.append(drawn["logp"])
        if t + 1 == max_new:
            break
        x = E[drawn["ids"].long()]
        q, k, v = policy.qkv(x)
        stage.write_cache(cache, k, v, slot(every, length + t).to(dev))
        seq_lens += 1
        out, _ = stage.decode(q, cache, device_table, seq_lens)
        h = policy.hidden(x, out)
    ids, logp = torch.stack(ids, 1), torch.stack(logp, 1)
    ended = (ids == end_id).cpu()
    n = torch.where(ended.any(1), ended.int().argmax(1) + 1, max_new)          # the end token is part of the response
    return dict(prompt_len=length, n=n, ids=[ids[b, :n[b]] for b in range(B)], logp=[logp[b, :n[b]] for b in range(B)],
                full=[torch.cat((prompts[b // group].to(dev), ids[b, :n[b]])) for b in range(B)])


def loss_and_gradients(policy, stage, loss_stage, batch, rewards, n_prompts, min_cut=1, seed=0, step=0):
    """The partial-token loss of the rollouts and its gradients with respect to every weight of the policy (float32)."""
    dev, w = stage.device, policy.weights
    B = len(batch["ids"])
    i32 = lambda t: t.to(torch.int32).to(dev)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64), batch["n"].cumsum(0))).to(dev)
    N = int(batch["n"].sum())
    ids = torch.cat(batch["ids"]).contiguous()
    adv = loss_stage.advantage(rewards.to(dev), n_prompts, B // n_prompts)
    kept = loss_stage.select_compact(nat.SelectParams(nat.RPC, min_cut=min_cut, seed=seed, step=step), cu, B, N, ids=ids,
                                     old_logp=torch.cat(batch["logp"]).contiguous())
    n_kept = kept["n_kept"]
    full = torch.cat(batch["full"]).contiguous()
    packed = loss_stage.prefix_pack(i32(batch["prompt_len"]), cu, kept["cut_len"], B, N, full.numel(), input_ids=full)
    rows, cu_rows = packed["total"], packed["cu_packed"]

    row_ids = packed["input_ids_packed"][:rows].long()
    x = w["E"][row_ids]
    q, k, v = policy.qkv(x)
    out, lse = stage.attention(q, k, v, cu_rows)
    h = policy.hidden(x, out)
    scored = packed["loss_row"][:n_kept].long()
    res = loss_stage.loss(h[scored], w["W"], kept["ids_k"], kept["old_logp_k"], adv, kept["kept_seq"], kept["kept_w"], n_kept)

    dh = torch.zeros_like(h)
    dh[scored] = res["dH"][:n_kept]                          # a row scores one token at most
    attended = out.view(rows, -1)
    dq, dk, dv = (g.view(rows, -1) for g in stage.attention_backward((dh @ w["Wo"].t()).view(out.shape), q, k, v, out, lse, cu_rows))
    dx = dh.float() + (dq @ w["Wq"].t()).float() + (dk @ w["Wk"].t()).float() + (dv @ w["Wv"].t()).float()
    grads = dict(E=torch.zeros(w["E"].shape, device=dev).index_add_(0, row_ids, dx), Wq=(x.t() @ dq).float(), Wk=(x.t() @ dk).float(),
                 Wv=(x.t() @ dv).float(), Wo=(attended.t() @ dh).float(), W=res["dW"])
    return dict(loss=res["loss"], grads=grads, logp=res["logp"][:n_kept], old_logp=kept["old_logp_k"][:n_kept], adv=adv, kept=kept, packed=packed)


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompts", type=int, default=8)
    ap.add_argument("--group", type=int, default=8)
    ap.add_argument("--max-new", type=int, default=64)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--q-heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--head-dim", type=int, default=64)
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--lr", type=float, default=10.0)
    ap.add_argument("--fp8", action="store_true", help="the cache in 8 bits")
    a = ap.parse_args(argv)
    policy = Policy(a.vocab, a.hidden, a.q_heads, a.kv_heads, a.head_dim)
    stage, loss_stage = RolloutStage(), LossStage()
    host = torch.Generator().manual_seed(1)
    words = torch.Generator(device=stage.device).manual_seed(2)
    for step in range(a.steps):
        prompts = [torch.randint(1, a.vocab, (int(n),), generator=host).to(torch.int32) for n in torch.randint(3, 40, (a.prompts,), generator=host)]
        batch = rollouts(policy, stage, prompts, a.group, a.max_new, fp8=a.fp8, generator=words)
        rewards = torch.stack([(r < a.vocab // 2).float().mean() for r in batch["ids"]])       # a preference that can be learned
        res = loss_and_gradients(policy, stage, loss_stage, batch, rewards, a.prompts, min_cut=8, seed=3, step=step)
        for name, g in res["grads"].items():
            policy.weights[name].sub_((a.lr * g).to(torch.bfloat16))
        gap = (res["logp"] - res["old_logp"]).abs()
        print(f"step {step}: reward {rewards.mean().item():.4f}  loss {res['loss'].item():+.4e}  kept {res['kept']['n_kept']} of {int(batch['n'].sum())} tokens"
              f"  |log-prob - behaviour log-prob| {gap.mean().item():.1e}")


if __name__ == "__main__":
    main()
