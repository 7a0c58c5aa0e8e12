"""One step of reinforcement learning with a small policy (embedding, one attention layer, head), every operator where it is used:

  rollouts   the prompts' embedding, norms and rotation of queries and keys (--rotate), attention over the packed prompts, pages of a cache for all rollouts and the
             prompts' keys and values into them; then token by token sampling, embedding, the next slots, cache write and attention over the cache.  The sampled
             tokens' log-probabilities are the behaviour log-probs of the loss;
  loss       advantages, random prefix cutting, the truncated batch, its embedding, norms, rotation and attention, the loss stage;
  gradients  of the head from the loss stage, of the layer through the attention's backward pass and that of norms and rotation, of the embedding, which with tied weights (--tied)
             is added to the head's.

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
    """h = x + attention(x Wq, x Wk, x Wv) Wo, x = E[ids]; logits = h W^T.  With rotate, queries and keys are normed head by head (weights Nq, Nk) and rotated by their
    positions; with tied, W is E."""

    def __init__(self, vocab, hidden, q_heads, kv_heads, head_dim, seed=0, device="cuda:0", rotate=False, tied=False):
        g = torch.Generator().manual_seed(seed)
        new = lambda rows, cols, std: (torch.randn(rows, cols, generator=g) * std).to(torch.bfloat16).to(device)
        self.q_heads, self.kv_heads, self.head_dim, self.rotate, self.tied = q_heads, kv_heads, head_dim, rotate, tied
        self.weights = dict(E=new(vocab, hidden, hidden ** -0.5 if tied else 1.0), Wq=new(hidden, q_heads * head_dim, hidden ** -0.5),
                            Wk=new(hidden, kv_heads * head_dim, hidden ** -0.5), Wv=new(hidden, kv_heads * head_dim, hidden ** -0.5),
                            Wo=new(q_heads * head_dim, hidden, (q_heads * head_dim) ** -0.5))
        self.scale = 4.0 if tied else 1.0            # of the embedding: rows of E have length 1, as the head wants them, and 1 would be little beside what attention adds
        if not tied:
            self.weights["W"] = new(vocab, hidden, hidden ** -0.5)
        self.inv_freq = None
        if rotate:
            self.weights.update(Nq=(1 + new(1, head_dim, 0.2)[0]), Nk=(1 + new(1, head_dim, 0.2)[0]))
            self.inv_freq = 1e4 ** (-2.0 * torch.arange(head_dim // 2, dtype=torch.float64, device=device) / head_dim)

    @property
    def head(self):
        return self.weights["E" if self.tied else "W"]

    def embed(self, stage, ids):
        return stage.embed(ids, self.weights["E"], self.scale)

    def qkv(self, stage, x, positions):
        """Queries, keys and values of rows x, and queries and keys as they were projected."""
        w, n = self.weights, x.shape[0]
        q, k, v = ((x @ w[name]).view(n, -1, self.head_dim) for name in ("Wq", "Wk", "Wv"))
        if not self.rotate:
            return q, k, v, (q, k)
        return *stage.norm_rotate(q, k, positions, self.inv_freq, w["Nq"], w["Nk"]), v, (q, k)

    def qk_backward(self, stage, dq, dk, projected, positions):
        """Gradients of what qkv() projected, and of the norms' weights."""
        if not self.rotate:
            return dq, dk, {}
        w = self.weights
        dq, dk, dnq, dnk = stage.norm_rotate_backward(dq, dk, *projected, positions, self.inv_freq, w["Nq"], w["Nk"])
        return dq, dk, dict(Nq=dnq, Nk=dnk)

    def hidden(self, x, attended):
        return x + attended.reshape(x.shape[0], -1) @ self.weights["Wo"]


def rollouts(policy, stage, prompts, group, max_new, page_size=16, fp8=False, temperature=1.0, top_p=1.0, end_id=0, generator=None, fp4=False):
    """`group` continuations of every prompt (a list of int32 id tensors), of up to max_new tokens, the last of them end_id or not.
    Returns per rollout: ids of prompt and response, response length, behaviour log-probs."""
    dev, W = stage.device, policy.head
    B = len(prompts) * group
    lens = torch.tensor([len(p) for p in prompts])
    cu = torch.cat((torch.zeros(1, dtype=torch.int64), lens.cumsum(0)))
    i32 = lambda t: t.to(torch.int32).to(dev)
    x = policy.embed(stage, torch.cat(prompts).to(dev))
    q, k, v, _ = policy.qkv(stage, x, i32(torch.cat([torch.arange(n) for n in lens])))
    out, _ = stage.attention(q, k, v, i32(cu))
    last = cu[1:] - 1
    h = policy.hidden(x, out)[last.to(dev)].repeat_interleave(group, 0)

    # pages of a rollout: as they come from the stack, which holds them in any order
    width = (int(lens.max()) + max_new + page_size - 1) // page_size
    cache = PagedCache.empty(B * width, policy.kv_heads, page_size, policy.head_dim, fp8=fp8, device=dev, fp4=fp4)
    table, free, counts = torch.full((B, width), -1, dtype=torch.int32, device=dev), i32(torch.randperm(B * width)), i32(torch.tensor([B * width, 0]))
    length = lens.repeat_interleave(group)
    rows = torch.cat([torch.arange(cu[b // group], cu[b // group + 1]) for b in range(B)]).to(dev)
    new = stage.reserve(table, torch.zeros(B, dtype=torch.int32, device=dev), i32(length), free, counts, page_size, rows.numel())
    stage.write_cache(cache, k[rows], v[rows], new["slots"])

    settings = dict(temperature=torch.full((B,), temperature, device=dev), top_p=torch.full((B,), top_p, device=dev))
    one_each = torch.ones(B, dtype=torch.int32, device=dev)
    ids, logp = [], []
    for t in range(max_new):
        word = torch.randint(-2 ** 31, 2 ** 31, (B,), dtype=torch.int32, device=dev, generator=generator)
        drawn = stage.sample(h @ W.t(), word, **settings)
        ids.append(drawn["ids"])
        logp.append(drawn["logp"])
        if t + 1 == max_new:
            break
        new = stage.reserve(table, new["seq_lens"], one_each, free, new["counts"], page_size, B)
        x = policy.embed(stage, drawn["ids"])
        q, k, v, _ = policy.qkv(stage, x, new["position_ids"])
        stage.write_cache(cache, k, v, new["slots"])
        out, _ = stage.decode(q, cache, table, new["seq_lens"])
        h = policy.hidden(x, out)
    _, counts = stage.release(table, new["seq_lens"], torch.zeros_like(one_each), free, new["counts"], page_size)
    ids, logp = torch.stack(ids, 1), torch.stack(logp, 1)
    ended = (ids == end_id).cpu()
    n = torch.where(ended.any(1), ended.int().argmax(1) + 1, max_new)          # the end token is part of the response
    return dict(prompt_len=length, n=n, ids=[ids[b, :n[b]] for b in range(B)], logp=[logp[b, :n[b]] for b in range(B)],
                full=[torch.cat((prompts[b // group].to(dev), ids[b, :n[b]])) for b in range(B)], free_pages=counts)


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

    row_ids, positions = packed["input_ids_packed"][:rows], packed["position_ids"][:rows]
    x = policy.embed(stage, row_ids)
    q, k, v, projected = policy.qkv(stage, x, positions)
    out, lse = stage.attention(q, k, v, cu_rows)
    h = policy.hidden(x, out)
    scored = packed["loss_row"][:n_kept].long()
    res = loss_stage.loss(h[scored], policy.head, kept["ids_k"], kept["old_logp_k"], adv, kept["kept_seq"], kept["kept_w"], n_kept)

    dh = torch.zeros_like(h)
    dh[scored] = res["dH"][:n_kept]                          # a row scores one token at most
    attended = out.view(rows, -1)
    dq, dk, dv = stage.attention_backward((dh @ w["Wo"].t()).view(out.shape), q, k, v, out, lse, cu_rows)
    dq, dk, norms = policy.qk_backward(stage, dq, dk, projected, positions)
    dq, dk, dv = (g.view(rows, -1) for g in (dq, dk, dv))
    dx = dh.float() + (dq @ w["Wq"].t()).float() + (dk @ w["Wk"].t()).float() + (dv @ w["Wv"].t()).float()
    dE = stage.embed_backward(dx, row_ids, w["E"].shape[0], policy.scale, dE=res["dW"] if policy.tied else None, accumulate=policy.tied)
    grads = dict(E=dE, Wq=(x.t() @ dq).float(), Wk=(x.t() @ dk).float(), Wv=(x.t() @ dv).float(), Wo=(attended.t() @ dh).float(), **norms)
    if not policy.tied:
        grads["W"] = res["dW"]
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
    ap.add_argument("--fp4", action="store_true", help="the cache in 4 bits")
    ap.add_argument("--rotate", action="store_true", help="queries and keys normed and rotated by position")
    ap.add_argument("--tied", action="store_true", help="one matrix for embedding and head")
    a = ap.parse_args(argv)
    policy = Policy(a.vocab, a.hidden, a.q_heads, a.kv_heads, a.head_dim, rotate=a.rotate, tied=a.tied)
    stage, loss_stage = RolloutStage(), LossStage()
    host = torch.Generator().manual_seed(1)
    words = torch.Generator(device=stage.device).manual_seed(2)
    for step in range(a.steps):
        prompts = [torch.randint(1, a.vocab, (int(n),), generator=host).to(torch.int32) for n in torch.randint(3, 40, (a.prompts,), generator=host)]
        batch = rollouts(policy, stage, prompts, a.group, a.max_new, fp8=a.fp8, fp4=a.fp4, generator=words)
        rewards = torch.stack([(r < a.vocab // 2).float().mean() for r in batch["ids"]])       # a preference that can be learned
        res = loss_and_gradients(policy, stage, loss_stage, batch, rewards, a.prompts, min_cut=8, seed=3, step=step)
        for name, g in res["grads"].items():
            policy.weights[name].sub_((a.lr * g).to(torch.bfloat16))
        gap = (res["logp"] - res["old_logp"]).abs()
        print(f"step {step}: reward {rewards.mean().item():.4f}  loss {res['loss'].item():+.4e}  kept {res['kept']['n_kept']} of {int(batch['n'].sum())} tokens"
              f"  |log-prob - behaviour log-prob| {gap.mean().item():.1e}")


if __name__ == "__main__":
    main()
