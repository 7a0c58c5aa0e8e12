"""Timed cases of the operators between token ids and attention: the embedding and its gradient, the norms and the rotation of queries
and keys, the block tables and slots of the paged cache, and the cache in 4 bits with the attention that reads it.

Where `own` is false, the operators are computed in their plain form: elementary torch operations, 32-bit arithmetic (64 for angles and
long sums), one rounding at the end.  Where it is true, the library's entry points compute them.
"""
import math
import random

import torch

own = False
_DEVICE = "cuda"
_stage = None
_GROUP = 32               # elements that share a power of two in the 4-bit format
_LARGEST = 6.0            # of the 4-bit format, 2 exponent bits and 1 mantissa bit
_EPS = 1e-6


def listed():
    return [
        # One decoding step: a token of each of 64 sequences, at places far apart.  Nothing but latency.
        {"name": "heads_step", "op": "heads", "n_seqs": 64, "max_q": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "rotary": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "cached": 40000},
        # The prompts of a batch.
        {"name": "heads_prompts", "op": "heads", "n_seqs": 6, "max_q": 4093, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "rotary": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "cached": 0},
        # Training step of a few short rollouts, small heads of which half the elements turn, in pairs of neighbours.
        {"name": "heads_train_short", "op": "heads_train", "n_seqs": 16, "max_q": 311, "q_heads": 16, "kv_heads": 16, "head_dim": 64, "rotary": 32,
         "interleaved": True, "norm": True, "dtype": "f32", "cached": 0},
        # Training step of a micro-batch of truncated rollouts of a response limit of 4096.
        {"name": "heads_train", "op": "heads_train", "n_seqs": 8, "max_q": 4096, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "rotary": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "cached": 0},
        # Token ids of the prompts of a batch into their rows.
        {"name": "embed_prompts", "op": "embed", "rows": 16381, "vocab": 151936, "hidden": 4096, "dtype": "bf16", "scale": 1.0},
        # Gradient of a small embedding: latency of the sort and of the sums of the frequent tokens.
        {"name": "embed_train_short", "op": "embed_train", "rows": 2897, "vocab": 32000, "hidden": 1024, "dtype": "f32", "scale": 32.0},
        # Gradient of a large vocabulary's embedding over a micro-batch: most of it is zeros that have to be written.
        {"name": "embed_train", "op": "embed_train", "rows": 20483, "vocab": 151936, "hidden": 4096, "dtype": "bf16", "scale": 1.0},
        # A decoding step of many rollouts: one new slot each, now and then a new page, and not enough of these for the last ones.
        {"name": "pages_step", "op": "pages", "n_seqs": 512, "max_len": 8192, "max_new": 1, "page": 64, "free": 0.5},
        # A batch that turns over: a third of the sequences end and give their pages back, a third begin with prompts, the others go on.
        {"name": "pages_turnover", "op": "pages", "n_seqs": 192, "max_len": 8192, "max_new": 4093, "page": 16, "free": 1.0},
        # New turns written behind cached conversations in 4 bits, and everything read back for their attention.
        {"name": "cache4_turns", "op": "cache4", "n_seqs": 6, "max_q": 701, "cached": 8191, "kv_heads": 4, "head_dim": 128, "page": 32},
        # One user, one long context, from the 4-bit cache.
        {"name": "decode4_single", "op": "decode4", "n_seqs": 1, "max_len": 32768, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "page": 64},
        # All rollouts of a few prompts at once, lengths far apart, from the 4-bit cache.
        {"name": "decode4_rollouts", "op": "decode4", "n_seqs": 128, "max_len": 8192, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["heads", "heads_train", "embed", "embed_train", "pages", "cache4", "decode4"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (16, 8), (16, 16), (16, 2), (12, 1)])
    head_dim = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("heads", "heads_train"):
        n_seqs = _log_int(rng, 1, 64)
        cached = _log_int(rng, 1, 100000) if op == "heads" and rng.random() < 0.4 else 0
        return {"op": op, "n_seqs": n_seqs, "max_q": _log_int(rng, 1, (8192 if dtype == "f32" else 16384) // n_seqs), "q_heads": q_heads,
                "kv_heads": kv_heads, "head_dim": head_dim, "rotary": rng.choice([head_dim, head_dim, head_dim // 2, 16]),
                "interleaved": rng.random() < 0.3, "norm": rng.random() < 0.8, "dtype": dtype, "cached": cached}
    if op in ("embed", "embed_train"):
        return {"op": op, "rows": _log_int(rng, 1, 20000), "vocab": rng.choice([151936, 152064, _log_int(rng, 2, 152064)]),
                "hidden": 8 * _log_int(rng, 8, 500), "dtype": dtype, "scale": rng.choice([1.0, 1.0, 22.5])}
    page = rng.choice([16, 32, 64, 128])
    if op == "pages":
        n_seqs = _log_int(rng, 1, 2048)
        max_new = 1 if rng.random() < 0.5 else _log_int(rng, 1, 4096)
        return {"op": op, "n_seqs": n_seqs, "max_len": _log_int(rng, 1, min(16384, 1500000 // n_seqs)),
                "max_new": max(1, min(max_new, 500000 // n_seqs)), "page": page, "free": rng.choice([0.5, 1.0])}
    if op == "cache4":
        n_seqs = _log_int(rng, 1, 32)
        return {"op": op, "n_seqs": n_seqs, "max_q": _log_int(rng, 1, 4096 // n_seqs), "cached": _log_int(rng, 1, 32768 // n_seqs),
                "kv_heads": kv_heads, "head_dim": head_dim, "page": page}
    n_seqs = _log_int(rng, 1, 128)
    return {"op": op, "n_seqs": n_seqs, "max_len": _log_int(rng, 1, min(40000, 300000 // n_seqs)), "q_heads": q_heads,
            "kv_heads": min(kv_heads, 8), "head_dim": head_dim, "page": page}


def _lengths(n, longest):
    """Lengths of n sequences, 1 .. longest, the first of them the longest: a wide spread, the same for every seed."""
    rng = random.Random(7919 * n + longest)
    return [longest] + [max(1, min(longest, int(longest * rng.uniform(0.15, 1.0)))) for _ in range(n - 1)]


def _cached_lengths(case):
    rng = random.Random(case["cached"] + 31)
    return [int(case["cached"] * rng.uniform(0.2, 1.0)) for _ in range(case["n_seqs"])]


def _page_lengths(case):
    """Per sequence: its length, what it keeps of it, and its new tokens.  Of a step, all have one; of a batch that turns over, a third end and a
    third, without any token so far, get a prompt."""
    have, new = _lengths(case["n_seqs"], case["max_len"]), _lengths(case["n_seqs"], case["max_new"])
    if case["max_new"] == 1:
        return have, have, [1] * len(have)
    part = [i % 3 for i in range(len(have))]
    have = [0 if p == 1 else n for p, n in zip(part, have)]
    return have, [0 if p == 0 else n for p, n in zip(part, have)], [0 if p == 0 else n if p == 1 else 1 for p, n in zip(part, new)]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=_DEVICE)


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32).to(_DEVICE)


def _pages_of(n, page):
    return -(-n // page)


def _block_table(lengths, page, width, generator, n_pages):
    """Pages of every sequence, in no order, behind one another in a table of `width`; unused places hold -1.  And the pages that are left."""
    order = torch.randperm(n_pages, generator=generator).to(torch.int32)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(lengths):
        need = _pages_of(n, page)
        table[i, :need] = order[at:at + need]
        at += need
    return table.to(_DEVICE), order[at:].to(_DEVICE)


def _token_ids(n, vocab, g):
    """Ids as text has them: a few tokens make up much of it.  A row in about 500 is padding (-1)."""
    u = torch.rand(n, generator=g, device=_DEVICE, dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab)).long().clamp(1, vocab) - 1
    ids = torch.randperm(vocab, generator=g, device=_DEVICE)[rank].to(torch.int32)
    return torch.where(torch.rand(n, generator=g, device=_DEVICE) < 0.002, -1, ids)


def prepare(case, seed):
    g = torch.Generator(device=_DEVICE).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    op = case["op"]
    state = dict(case)
    dtype = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    normal = lambda *shape: torch.randn(shape, generator=g, device=_DEVICE, dtype=dtype)  # noqa: E731
    if op in ("heads", "heads_train"):
        lengths = _lengths(case["n_seqs"], case["max_q"])
        n, hq, hkv, D = sum(lengths), case["q_heads"], case["kv_heads"], case["head_dim"]
        qkv = normal(n, hq + 2 * hkv, D)                    # of one projection
        qkv *= torch.exp(0.5 * torch.randn((n, hq + 2 * hkv, 1), generator=g, device=_DEVICE)).to(dtype)
        state["q"], state["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]
        state["q_weight"], state["k_weight"] = ((1.0 + 0.2 * normal(D)).to(dtype) if case["norm"] else None for _ in range(2))
        before = [0] * len(lengths) if not case["cached"] else torch.randint(case["cached"], (len(lengths),), generator=host).tolist()
        state["position_ids"] = torch.cat([torch.arange(b, b + t, dtype=torch.int32) for b, t in zip(before, lengths)]).to(_DEVICE)
        half = torch.arange(case["rotary"] // 2, dtype=torch.float64, device=_DEVICE)
        state["inv_freq"] = 1e6 ** (-2.0 * half / case["rotary"])
        if op == "heads_train":
            state["dq_out"], state["dk_out"] = normal(n, hq, D), normal(n, hkv, D)
    elif op in ("embed", "embed_train"):
        state["ids"] = _token_ids(case["rows"], case["vocab"], g)
        if op == "embed":
            state["table"] = 0.02 * normal(case["vocab"], case["hidden"])
        else:
            state["dout"] = normal(case["rows"], case["hidden"])
    elif op == "pages":
        have, keep, new = _page_lengths(case)
        page = case["page"]
        width = max(_pages_of(h + x, page) for h, x in zip(have, new))
        used = sum(_pages_of(h, page) for h in have)
        need = sum(_pages_of(k + x, page) - _pages_of(k, page) for k, x in zip(keep, new))
        back = sum(_pages_of(h, page) - _pages_of(k, page) for h, k in zip(have, keep))
        left = max(0, int(case["free"] * need) - back)
        n_pages = used + left + back + 3
        state["block_table"], rest = _block_table(have, page, width, host, n_pages)
        state["free_pages"] = torch.full((n_pages,), -1, dtype=torch.int32, device=_DEVICE)
        state["free_pages"][:left] = rest[:left]
        state["counts"] = _i32([left, 0])
        state["seq_lens"], state["keep_lens"], state["new_lens"] = _i32(have), _i32(keep), _i32(new)
        state["n_rows"], state["turns"] = sum(new), keep != have
    else:
        if op == "cache4":
            before, new = _cached_lengths(case), _lengths(case["n_seqs"], case["max_q"])
            lengths = [a + b for a, b in zip(before, new)]
        else:
            lengths = _lengths(case["n_seqs"], case["max_len"])
        page, hkv, D = case["page"], case["kv_heads"], case["head_dim"]
        n_pages = sum(_pages_of(n, page) for n in lengths) + 2
        state["block_table"], _ = _block_table(lengths, page, max(_pages_of(n, page) for n in lengths), host, n_pages)
        for name in ("k", "v"):
            x = normal(n_pages, hkv, page, D)
            state[name + "_cache"], state[name + "_exp"] = _quantise(x.float())
        state["cu_k"], state["n_total"], state["max_k"] = _offsets(lengths), sum(lengths), max(lengths)
        if op == "cache4":
            size = torch.exp(torch.randn((sum(new), 1, 1), generator=g, device=_DEVICE))       # rows of very different size
            state["k"], state["v"] = (normal(sum(new), hkv, D) * size).to(dtype), normal(sum(new), hkv, D)
            seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
            at = torch.cat([torch.arange(b, b + t) for b, t in zip(before, new)])
            state["slots"] = state["block_table"][seq.to(_DEVICE), (at // page).to(_DEVICE)].long() * page + (at % page).to(_DEVICE)
        else:
            state["seq_lens"] = _i32(lengths)
            state["q"] = normal(case["n_seqs"], case["q_heads"], D)
    return state


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _turned(x, position_ids, inv_freq, interleaved, sign):
    """x [rows, heads, D] with the pairs of its first 2 * len(inv_freq) elements turned by sign * position * inv_freq."""
    angle = (sign * position_ids.double())[:, None] * inv_freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    R = 2 * inv_freq.numel()
    turning, rest = x[..., :R], x[..., R:]
    a, b = (turning[..., 0::2], turning[..., 1::2]) if interleaved else (turning[..., :R // 2], turning[..., R // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1)


def _plain_heads(st, name):
    x, w = st[name].float(), st[name + "_weight"]
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w.float()
    return _turned(x, st["position_ids"], st["inv_freq"], st["interleaved"], 1).to(st[name].dtype)


def _plain_heads_backward(st, name):
    x, w = st[name].float(), st[name + "_weight"]
    dn = _turned(st["d" + name + "_out"].float(), st["position_ids"], st["inv_freq"], st["interleaved"], -1)
    if w is None:
        return dn.to(st[name].dtype), None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
    unit = x * r
    dw = (dn * unit).sum((0, 1), dtype=torch.float64).float()
    dn = dn * w.float()
    return (r * (dn - unit * (dn * unit).mean(-1, keepdim=True))).to(st[name].dtype), dw


def _plain_embed(st):
    ids, E = st["ids"].long(), st["table"]
    there = (ids >= 0) & (ids < E.shape[0])
    rows = E[torch.where(there, ids, 0)].float() * st["scale"]
    return torch.where(there[:, None], rows, 0.0).to(E.dtype)


def _plain_embed_backward(st):
    ids, V = st["ids"].long(), st["vocab"]
    there = (ids >= 0) & (ids < V)
    sums = torch.zeros((V + 1, st["hidden"]), dtype=torch.float32, device=ids.device)
    sums.index_add_(0, torch.where(there, ids, V), st["dout"].float())
    return sums[:V] * st["scale"]


def _whole(n, page):
    return (n + page - 1) // page


def _plain_release(st):
    """The pages behind what each sequence keeps, in order of sequence and place, onto the stack of free pages."""
    page, table, lens = st["page"], st["block_table"], st["seq_lens"].long()
    kept = torch.minimum(lens, st["keep_lens"].long())
    place = torch.arange(table.shape[1], device=table.device)
    back = (place >= _whole(kept, page)[:, None]) & (place < _whole(lens, page)[:, None])
    left = st["counts"][0].long()
    count = back.sum()
    to = left + back.flatten().cumsum(0) - 1
    free = st["free_pages"]
    # entries that do not go back are written behind the stack's end, into a place that is cut off
    padded = torch.cat((free, free[:1]))
    padded[torch.where(back.flatten(), to, free.numel())] = table.flatten()
    free.copy_(padded[:-1])
    return kept, left + count


def _plain_pages(st):
    page, table, free, new = st["page"], st["block_table"], st["free_pages"], st["new_lens"].long()
    out = {}
    lens, left = st["seq_lens"].long(), st["counts"][0].long()
    if st["turns"]:
        lens, left = _plain_release(st)
    first = _whole(lens, page)
    need = _whole(lens + new, page) - first
    running = need.cumsum(0)
    served = (need == 0) | (running <= left)
    cu = torch.cat((torch.zeros_like(new[:1]), new.cumsum(0)))
    row = torch.arange(st["n_rows"], device=new.device)
    seq = torch.bucketize(row, cu[1:], right=True)
    at = lens[seq] + row - cu[seq]
    # new pages: from the top of the stack, sequence by sequence
    place = torch.arange(table.shape[1], device=table.device)
    fresh = served[:, None] & (place >= first[:, None]) & (place < (first + need)[:, None])
    which = left - 1 - ((running - need)[:, None] + place - first[:, None])
    table.copy_(torch.where(fresh, free[which.clamp(0, free.numel() - 1)], table))
    slots = table[seq, at // page].long() * page + at % page
    out["slots"] = torch.where(served[seq], slots, -1)
    out["position_ids"], out["cu_new"], out["start"] = at.int(), cu.int(), torch.where(served, lens, -1).int()
    out["seq_lens"] = (lens + torch.where(served, new, 0)).int()
    out["counts"] = torch.stack((left - torch.where(served, need, 0).sum(), (~served).sum())).int()
    return {**out, "block_table": table, "free_pages": free}


def _quantise(x):
    """Groups of 32 elements in 4 bits with one power of two each, the smallest that brings the largest magnitude to 6 or less (2^-125 at
    least); two elements to a byte, the first in its low half."""
    shape = x.shape
    x = x.reshape(*shape[:-1], -1, _GROUP)
    mantissa, e = torch.frexp(x.abs().amax(-1) / _LARGEST)       # mantissa in [1/2, 1): the power of two above it, or equal
    e = torch.where(mantissa == 0.5, e - 1, e).clamp(-125, 127)
    e = torch.where(mantissa == 0, -125, e)
    y = torch.ldexp(x, -e[..., None])
    m = y.abs()
    code = (m > 0.25).to(torch.uint8)                            # 0, 1/2, 1, 3/2, 2, 3, 4, 6; halfway the even code
    for border, even in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (m >= border) if even else (m > border)
    code += 8 * torch.signbit(x).to(torch.uint8)
    code = code.view(shape)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _values(codes, exponents):
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    x = torch.where(both >= 8, -grid[both & 7], grid[both & 7])
    e = exponents.to(torch.int32)[..., None] - 127
    return torch.ldexp(x.view(*e.shape[:-1], _GROUP), e).view(x.shape)


def _places(cu, n_rows):
    """Sequence and position of every packed row."""
    row = torch.arange(n_rows, device=cu.device)
    seq = torch.bucketize(row, cu[1:].long(), right=True)
    return seq, row - cu[seq].long()


def _cached_rows(st, name, seq, at):
    """Rows (seq, at) of a cache in 32 bits: [rows..., heads, D]."""
    pages = st["block_table"][seq, at // st["page"]].clamp(min=0).long()
    return _values(st[name + "_cache"][pages, :, at % st["page"]], st[name + "_exp"][pages, :, at % st["page"]])


def _plain_cache4(st):
    slots, page = st["slots"], st["page"]
    for name in ("k", "v"):
        codes, e = _quantise(st[name].float())
        st[name + "_cache"][slots // page, :, slots % page] = codes
        st[name + "_exp"][slots // page, :, slots % page] = e
    seq, at = _places(st["cu_k"], st["n_total"])
    return {name: _cached_rows(st, name, seq, at).bfloat16() for name in ("k", "v")}


def _plain_decode4(st):
    q = st["q"]
    S, hq, D = q.shape
    hkv = st["kv_heads"]
    at = torch.arange(st["max_k"], device=q.device).expand(S, -1)
    seq = torch.arange(S, device=q.device)[:, None].expand_as(at)
    kp, vp = (_cached_rows(st, name, seq, at).permute(0, 2, 1, 3).contiguous() for name in ("k", "v"))
    s = torch.matmul(q.float().view(S, hkv, hq // hkv, D), kp.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D))
    s.masked_fill_(at[:, None, None] >= st["seq_lens"][:, None, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    return {"out": torch.matmul(p.div_(total), vp).reshape(S, hq, D).to(q.dtype), "lse": (m + total.log()).reshape(S, hq)}


# ---- the library's entry points ------------------------------------------------------------------------------------------

def _own(st):
    global _stage
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    if _stage is None:
        _stage = RolloutStage(_DEVICE)
    op = st["op"]
    if op in ("heads", "heads_train"):
        how = dict(q_weight=st["q_weight"], k_weight=st["k_weight"], eps=_EPS, interleaved=st["interleaved"])
        q, k = _stage.norm_rotate(st["q"], st["k"], st["position_ids"], st["inv_freq"], **how)
        if op == "heads":
            return {"q": q, "k": k}
        dq, dk, dqw, dkw = _stage.norm_rotate_backward(st["dq_out"], st["dk_out"], st["q"], st["k"], st["position_ids"], st["inv_freq"], **how)
        return {"q": q, "k": k, "dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
    if op == "embed":
        return _stage.embed(st["ids"], st["table"], st["scale"])
    if op == "embed_train":
        return _stage.embed_backward(st["dout"], st["ids"], st["vocab"], st["scale"])
    if op == "pages":
        lens, counts = st["seq_lens"], st["counts"]
        if st["turns"]:
            lens, counts = _stage.release(st["block_table"], lens, st["keep_lens"], st["free_pages"], counts, st["page"])
        out = _stage.reserve(st["block_table"], lens, st["new_lens"], st["free_pages"], counts, st["page"], st["n_rows"])
        return {**out, "block_table": st["block_table"], "free_pages": st["free_pages"]}
    cache = PagedCache(st["k_cache"], st["v_cache"], st["k_exp"], st["v_exp"])
    if op == "cache4":
        _stage.write_cache(cache, st["k"], st["v"], st["slots"])
        k, v = _stage.read_cache(cache, st["block_table"], st["cu_k"], st["n_total"])
        return {"k": k, "v": v}
    out, lse = _stage.decode(st["q"], cache, st["block_table"], st["seq_lens"])
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _own(state)
    op = state["op"]
    if op in ("heads", "heads_train"):
        out = {name: _plain_heads(state, name) for name in ("q", "k")}
        if op == "heads_train":
            for name in ("q", "k"):
                out["d" + name], out["d" + name + "_weight"] = _plain_heads_backward(state, name)
        return out
    return {"embed": _plain_embed, "embed_train": _plain_embed_backward, "pages": _plain_pages, "cache4": _plain_cache4,
            "decode4": _plain_decode4}[op](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    size = 4 if case.get("dtype") == "f32" else 2
    if op in ("heads", "heads_train"):
        rows = sum(_lengths(case["n_seqs"], case["max_q"]))
        values = rows * (case["q_heads"] + case["kv_heads"]) * case["head_dim"]
        passes = 2 if op == "heads" else 5                  # rows in and out; and gradients, rows, gradients
        return {"bytes": passes * values * size + 4 * rows, "flops": (8 if op == "heads" else 24) * values}
    if op in ("embed", "embed_train"):
        values = case["rows"] * case["hidden"]
        if op == "embed":
            return {"bytes": 2 * values * size + 4 * case["rows"], "flops": values}
        return {"bytes": values * size + 4 * case["vocab"] * case["hidden"] + 4 * case["rows"], "flops": values}
    if op == "pages":
        have, keep, new = _page_lengths(case)
        page = case["page"]
        need = sum(_pages_of(k + x, page) - _pages_of(k, page) for k, x in zip(keep, new))
        back = sum(_pages_of(h, page) - _pages_of(k, page) for h, k in zip(have, keep))
        return {"bytes": 12 * sum(new) + 8 * (need + back) + 24 * len(have), "flops": 0}
    row = case["head_dim"] // 2 + case["head_dim"] // _GROUP
    if op == "cache4":
        before, new = sum(_cached_lengths(case)), sum(_lengths(case["n_seqs"], case["max_q"]))
        written, read = new * (2 * case["head_dim"] + row), (before + new) * (2 * case["head_dim"] + row)
        return {"bytes": 2 * case["kv_heads"] * (written + read) + 8 * new, "flops": 0}
    lengths = _lengths(case["n_seqs"], case["max_len"])
    n, rows = sum(lengths), case["n_seqs"] * case["q_heads"]
    return {"bytes": 2 * n * case["kv_heads"] * row + 4 * sum(_pages_of(t, case["page"]) for t in lengths) + rows * (4 * case["head_dim"] + 4),
            "flops": 4 * n * case["q_heads"] * case["head_dim"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def _exact_heads(x, w, position_ids, inv_freq, interleaved):
    """As products of complex numbers, in 64 bits each part; differentiable."""
    if w is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + _EPS) * w
    R = 2 * inv_freq.numel()
    turn = torch.exp(1j * (position_ids.double()[:, None] * inv_freq))[:, None]
    pairs = x[..., :R].unflatten(-1, (R // 2, 2) if interleaved else (2, R // 2))
    z = (torch.complex(pairs[..., 0], pairs[..., 1]) if interleaved else torch.complex(pairs[..., 0, :], pairs[..., 1, :])) * turn
    parts = torch.view_as_real(z)
    return torch.cat((parts.flatten(-2) if interleaved else parts.transpose(-1, -2).flatten(-2), x[..., R:]), -1)


def _exact_all_heads(st):
    out = {}
    for name in ("q", "k"):
        leaf = st[name].double().requires_grad_(st["op"] == "heads_train")
        w = None if st[name + "_weight"] is None else st[name + "_weight"].double().requires_grad_(st["op"] == "heads_train")
        y = _exact_heads(leaf, w, st["position_ids"], st["inv_freq"], st["interleaved"])
        out[name] = y.detach()
        if st["op"] == "heads_train":
            y.backward(st["d" + name + "_out"].double())
            out["d" + name], out["d" + name + "_weight"] = leaf.grad, None if w is None else w.grad
    return out


def _exact_embed_backward(st):
    """Sums over runs of equal ids in sorted order, as differences of running sums, some columns at a time."""
    ids = st["ids"].long()
    ids, order = torch.sort(ids, stable=True)
    keep = (ids >= 0) & (ids < st["vocab"])
    ids, order = ids[keep], order[keep]
    out = torch.zeros((st["vocab"], st["hidden"]), dtype=torch.float64, device=ids.device)
    if ids.numel() == 0:
        return out
    last = torch.cat(((ids[1:] != ids[:-1]).nonzero()[:, 0], torch.tensor([ids.numel() - 1], device=ids.device)))
    for c in range(0, st["hidden"], 512):
        running = st["dout"][order, c:c + 512].double().cumsum(0)[last]
        out[ids[last], c:c + 512] = torch.diff(running, dim=0, prepend=torch.zeros_like(running[:1])) * st["scale"]
    return out


def _exact_pages(st):
    """Sequence by sequence, page by page."""
    page = st["page"]
    table, free, lens = st["block_table"].tolist(), st["free_pages"].tolist(), st["seq_lens"].tolist()
    left, pages = st["counts"][0].item(), lambda n: -(-n // page)
    if st["turns"]:
        for i, keep in enumerate(st["keep_lens"].tolist()):
            for place in range(pages(min(keep, lens[i])), pages(lens[i])):
                free[left] = table[i][place]
                left += 1
            lens[i] = min(keep, lens[i])
    top, asked, refused = left, 0, 0
    cu, start, slots, at = [0], [], [], []
    for i, new in enumerate(st["new_lens"].tolist()):
        places = range(pages(lens[i]), pages(lens[i] + new))
        asked += len(places)
        served = not places or asked <= top
        for place in places if served else ():
            left -= 1
            table[i][place] = free[left]
        refused += not served
        cu.append(cu[-1] + new)
        start.append(lens[i] if served else -1)
        at += range(lens[i], lens[i] + new)
        slots += [table[i][t // page] * page + t % page if served else -1 for t in range(lens[i], lens[i] + new)]
        lens[i] += new if served else 0
    return {"slots": torch.tensor(slots, dtype=torch.int64, device=_DEVICE), "position_ids": _i32(at), "cu_new": _i32(cu), "start": _i32(start),
            "seq_lens": _i32(lens), "counts": _i32([left, refused]), "block_table": _i32(table), "free_pages": _i32(free)}


def _exact_cached(st, name, seq, length):
    at = torch.arange(length, device=_DEVICE)
    pages = st["block_table"][seq].long()[at // st["page"]]
    codes, e = st[name + "_cache"][pages, :, at % st["page"]].long(), st[name + "_exp"][pages, :, at % st["page"]]
    codes = torch.stack((codes % 16, codes // 16), -1).flatten(-2)
    low, high = (codes % 2).double(), (codes // 2 % 4).double()
    size = torch.where(high == 0, 0.5 * low, (1.0 + 0.5 * low) * torch.exp2(high - 1.0))
    return torch.where(codes >= 8, -size, size) * torch.exp2(e.double() - 127.0).repeat_interleave(_GROUP, -1)


def _exact_groups(x):
    """The value that the 4-bit format stands for instead of each element: the nearest of its list, of two as near the one with the even code."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    y = x.double().unflatten(-1, (-1, _GROUP))
    largest = y.abs().amax(-1, keepdim=True)
    e = torch.where(largest > 0, torch.ceil(torch.log2(largest / 6.0) - 1e-13), -125.0).clamp(min=-125.0)
    m = y.abs() * torch.exp2(-e)
    off = (m[..., None] - grid).abs()
    off += 1e-9 * (torch.arange(8, device=x.device) % 2)
    return (torch.copysign(grid[off.argmin(-1)], y) * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("heads", "heads_train"):
        return _exact_all_heads(st)
    if op == "embed":
        ids = st["ids"].long()
        there = ((ids >= 0) & (ids < st["vocab"]))[:, None]
        return torch.where(there, st["table"].double()[ids.clamp(min=0)] * st["scale"], 0.0)
    if op == "embed_train":
        return _exact_embed_backward(st)
    if op == "pages":
        return _exact_pages(st)
    lengths = torch.diff(st["cu_k"]).tolist()
    if op == "cache4":
        new, out = _lengths(case["n_seqs"], case["max_q"]), {}
        for name in ("k", "v"):
            written = _exact_groups(st[name]).split(new)
            out[name] = torch.cat([torch.cat((_exact_cached(st, name, i, n - new[i]), written[i])) for i, n in enumerate(lengths)])
        return out
    out, lse = [], []
    G = case["q_heads"] // case["kv_heads"]
    for i, n in enumerate(lengths):
        k, v = _exact_cached(st, "k", i, n), _exact_cached(st, "v", i, n)
        q = st["q"][i].double().view(case["kv_heads"], G, -1)
        s = torch.einsum("hgd,nhd->hgn", q, k) / math.sqrt(case["head_dim"])
        lse.append(torch.logsumexp(s, -1).reshape(-1))
        out.append(torch.einsum("hgn,nhd->hgd", torch.softmax(s, -1), v).reshape(case["q_heads"], -1))
    return {"out": torch.stack(out), "lse": torch.stack(lse)}
