"""Buffer plumbing around the operators of the model body and of the rollouts: the embedding, norms and rotation of queries and keys, attention
over packed sequences, and their gradients; a paged key-value cache, its pages, attention of one new token over it, sampling.  Outputs and workspaces come from torch;
the work happens in the library, on the current stream."""
import math

import torch

from . import binding as nb


class PagedCache(nb.KvCache):
    """A KvCache that can allocate its arrays."""

    @classmethod
    def empty(cls, n_pages, n_kv_heads, page_size, head_dim, fp8=False, device="cuda:0", fp4=False):
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        new = lambda s, dt: torch.empty(s, dtype=dt, device=device)
        if fp8 and fp4:
            raise ValueError("a cache is in 8 bits or in 4")
        if fp4:
            half, exps = (*shape[:3], head_dim // 2), (*shape[:3], head_dim // 32)
            return cls(new(half, torch.uint8), new(half, torch.uint8), new(exps, torch.uint8), new(exps, torch.uint8))
        dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
        exps = (new(shape[:3], torch.uint8), new(shape[:3], torch.uint8)) if fp8 else (None, None)
        return cls(new(shape, dt), new(shape, dt), *exps)


class RolloutStage:
    """Inputs may have any row stride that the library takes, and may be expanded along their rows (a gradient that is equal for all rows, one prompt's logits for a
    group of continuations): these are copied.

    Outputs are allocated, not cleared: rows of q (and out, dq, ...) or of k that belong to no sequence, in front of cu[0] or behind cu[-1], are left as the
    allocator gave them, NaN included.  With arrays that are longer than their sequences cut the results, or clear these rows, before a product sums over all.

    Attention and decoding take products in bf16 with fp32 sums: the probabilities (and the gradients dS) are rounded to bf16 before the second product (from a cache in 4 bits to
    16 bits), see nat.h."""

    def __init__(self, device="cuda:0"):
        self.device = torch.device(device)
        self._ws = {}

    def _buf(self, key, nbytes):
        """Workspace, kept per stream: calls on one stream follow one another, calls on different streams may overlap.  A call that is being recorded gets one of its
        own, from the graph's memory: a graph keeps the address, and its replays follow neither the later calls of this stream nor other graphs recorded on it."""
        if nbytes == 0:
            return None
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(int(nbytes), dtype=torch.uint8, device=self.device)
        key = (key, nb._stream())
        t = self._ws.get(key)
        if t is None or t.numel() < nbytes:
            t = self._ws[key] = torch.empty(int(nbytes), dtype=torch.uint8, device=self.device)
        return t

    @staticmethod
    def _scale(scale, head_dim):
        return 1.0 / math.sqrt(head_dim) if scale is None else scale

    def attention(self, q, k, v, cu_q, cu_k=None, causal=True, scale=None):
        """q [n_q, q heads, D], k, v [n_k, kv heads, D] bf16, packed by the int32 offsets cu_q, cu_k (None: the same).
        Returns (out like q, log-sum-exp [q heads, n_q]); rows of no sequence are not written."""
        out = torch.empty_like(q)                    # (half the host time of torch.empty; rows back to back whatever those of q)
        lse = q.new_empty((q.shape[1], q.shape[0]), dtype=torch.float32)
        ws = self._buf("attn_fwd", nb.attn_fwd_workspace_bytes(q.shape[0], k.shape[0], cu_q.numel() - 1, q.shape[1], k.shape[1], q.shape[2], causal))
        nb.nat_attn_fwd(q, k, v, cu_q, cu_q if cu_k is None else cu_k, causal, self._scale(scale, q.shape[2]), out, lse, ws)
        return out, lse

    def attention_backward(self, dout, q, k, v, out, lse, cu_q, cu_k=None, causal=True, scale=None):
        """(dq, dk, dv) of attention(), with its results; rows of no sequence are not written."""
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        ws = self._buf("attn_bwd", nb.attn_bwd_workspace_full_bytes(q.shape[0], k.shape[0], cu_q.numel() - 1, q.shape[1], k.shape[1], q.shape[2], causal))
        nb.nat_attn_bwd(q, k, v, out, lse, dout, cu_q, cu_q if cu_k is None else cu_k, causal, self._scale(scale, q.shape[2]),
                        dq, dk, dv, ws)
        return dq, dk, dv

    def norm_rotate(self, q, k, position_ids, inv_freq, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
        """Queries [n, q heads, D] and keys [n, kv heads, D], bf16 or float32, normed head by head (where there is a weight [D]) and rotated by position:
        inv_freq float64 [R / 2], radians per position for the pairs of the first R elements; both None: no rotation.  Returns (q, k), new arrays."""
        p, q, k, at = nb._qk_params(q, k, q_weight, k_weight, position_ids, inv_freq, eps, interleaved)
        q_out, k_out = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
        nb._qk_forward(p, q, k, at, q_out, k_out, (q_weight, k_weight, position_ids, inv_freq))
        return q_out, k_out

    def norm_rotate_backward(self, dq_out, dk_out, q, k, position_ids, inv_freq, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
        """(dq, dk, dq_weight, dk_weight) of norm_rotate() with its inputs; the weights' in float32, None without a weight."""
        p, q, k, at = nb._qk_params(q, k, q_weight, k_weight, position_ids, inv_freq, eps, interleaved)
        dq, dk = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
        dqw, dkw = (None if w is None else torch.empty_like(w, dtype=torch.float32) for w in (q_weight, k_weight))
        ws = None
        if dqw is not None or dkw is not None:
            ws = self._buf("norm_rotate", nb.qk_norm_rope_bwd_workspace_bytes(p.n_rows, p.head_dim))
        nb._qk_backward(p, q, k, at, dq_out, dk_out, dq, dk, dqw, dkw, 0, ws, (q_weight, k_weight, position_ids, inv_freq))
        return dq, dk, dqw, dkw

    def embed(self, ids, E, scale=1.0):
        """Rows of E [V, H] (bf16 or float32) by int32 ids, times scale; zeros for ids outside [0, V)."""
        out = E.new_empty((ids.numel(), E.shape[1]))
        nb.nat_embed(ids, E, scale, out)
        return out

    def embed_backward(self, dout, ids, V, scale=1.0, dE=None, accumulate=False):
        """The gradient [V, H] of embed(), float32; with accumulate it is added to dE (of tied weights: the head's dW)."""
        if dE is None:
            if accumulate:
                raise ValueError("accumulate needs dE")
            dE = dout.new_empty((V, dout.shape[1]), dtype=torch.float32)
        elif dE.shape[0] != V:
            raise ValueError(f"dE: expected {V} rows, got {dE.shape[0]}")
        ws = self._buf("embed", nb.embed_bwd_workspace_bytes(ids.numel(), V, dout.shape[1]))
        nb.nat_embed_bwd(ids, dout, scale, dE, accumulate, ws)
        return dE

    def reserve(self, block_table, seq_lens, new_lens, free_pages, counts, page_size, n_rows):
        """Pages for new_lens more tokens of every sequence, from the end of the stack free_pages[:counts[0]] into block_table (in place), and the places of these tokens:
        dict with slots (int64) and position_ids (int32) of the n_rows new rows, cu_new (their offsets), start (first position; -1: refused, no pages or no
        room in the table), and seq_lens and counts (free pages, sequences refused) as they are now.  The free pages stay where they are, behind counts[0]."""
        args = nb._pages_args(block_table, seq_lens, new_lens, "new_lens", free_pages, counts, page_size)
        n = args[2]
        ws_bytes = nb.kv_reserve_workspace_bytes(n)
        used = 3 * n + 3 + n_rows
        rest = -used % 64 + ws_bytes // 4                  # the workspace behind the results, at the next 256 bytes
        whole = torch.empty(used + rest, dtype=torch.int32, device=seq_lens.device)
        slots = torch.empty(n_rows, dtype=torch.int64, device=seq_lens.device)
        at = whole.data_ptr()
        cu, start, lens, pos = at + 8, at + 12 + 4 * n, at + 12 + 8 * n, at + 12 + 12 * n
        nb._reserve(args, n_rows, at, lens, start, cu, slots.data_ptr(), pos, at + 4 * (used + rest) - ws_bytes, ws_bytes)
        left, cu, start, lens, pos, _ = whole.split((2, n + 1, n, n, n_rows, rest))
        return dict(slots=slots, position_ids=pos, cu_new=cu, start=start, seq_lens=lens, counts=left)

    def release(self, block_table, seq_lens, keep_lens, free_pages, counts, page_size):
        """The pages behind the first keep_lens tokens of every sequence (0: it has ended) back to free_pages (in place): (seq_lens, counts) as they are now.
        A page goes back once for each row that has it there: of rows that share pages all but one must have -1 in their places."""
        args = nb._pages_args(block_table, seq_lens, keep_lens, "keep_lens", free_pages, counts, page_size)
        n = args[2]
        ws_bytes = nb.kv_release_workspace_bytes(n)
        rest = -(n + 2) % 64 + ws_bytes // 4
        whole = torch.empty(n + 2 + rest, dtype=torch.int32, device=seq_lens.device)
        at = whole.data_ptr()
        nb._release(args, at, at + 8, at + 4 * (n + 2 + rest) - ws_bytes, ws_bytes)
        left, lens, _ = whole.split((2, n, rest))
        return lens, left

    def write_cache(self, cache, k, v, slots):
        nb.nat_kv_write(cache, k, v, slots)

    def read_cache(self, cache, block_table, cu_k, n_rows):
        """The first cu_k[b + 1] - cu_k[b] tokens of every sequence as packed bf16 rows: (k, v)."""
        shape = (n_rows, cache.n_kv_heads, cache.head_dim)
        k, v = cache.k.new_empty(shape, dtype=torch.bfloat16), cache.k.new_empty(shape, dtype=torch.bfloat16)
        nb.nat_kv_read(cache, block_table, cu_k, k, v)
        return k, v

    def decode(self, q, cache, block_table, seq_lens, scale=None):
        """Attention of one token per sequence, q [n_seqs, q heads, D], over its cached tokens: (out like q, log-sum-exp [n_seqs, q heads])."""
        n, hq, dim = q.shape
        out = torch.empty_like(q)
        lse = q.new_empty((n, hq), dtype=torch.float32)
        ws = self._buf("decode", nb.attn_decode_workspace_bytes(n, hq, cache.n_kv_heads, cache.head_dim,
                                                               block_table.shape[1] * cache.page_size))
        nb.nat_attn_decode(cache, q, block_table, seq_lens, self._scale(scale, dim), out, lse, ws)
        return out, lse

    def sample(self, logits, random, temperature=None, top_k=None, top_p=None, min_p=None):
        """The next token of every row, its log-probability under the soft-max of the logits (the behaviour log-prob), and under
        the filtered distribution that it was drawn from: dict with ids, logp, logq."""
        n = logits.shape[0]
        new = lambda dt: logits.new_empty(n, dtype=dt)
        out = dict(ids=new(torch.int32), logp=new(torch.float32), logq=new(torch.float32))
        ws = self._buf("sample", nb.sample_workspace_bytes(n, logits.shape[1], nb._dtype_code(logits)))
        nb.nat_sample(logits, random, temperature, top_k, top_p, min_p, out["ids"], out["logp"], out["logq"], ws)
        return out
