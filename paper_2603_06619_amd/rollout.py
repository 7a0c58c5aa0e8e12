"""Buffer plumbing around the operators of the model body and of the rollouts: attention over packed sequences and its
gradients, a paged key-value cache, attention of one new token over it, sampling.  Outputs and workspaces come from torch;
the work happens in the library, on the current stream."""
import math

import torch

from . import binding as nb


class PagedCache(nb.KvCache):
    """A KvCache that can allocate its arrays."""

    @classmethod
    def empty(cls, n_pages, n_kv_heads, page_size, head_dim, fp8=False, device="cuda:0"):
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        new = lambda s, dt: torch.empty(s, dtype=dt, device=device)
        dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
        exps = (new(shape[:3], torch.uint8), new(shape[:3], torch.uint8)) if fp8 else (None, None)
        return cls(new(shape, dt), new(shape, dt), *exps)


class RolloutStage:
    """Inputs may have any row stride that the library takes, and may be expanded along their rows (a gradient that is equal for all rows, one prompt's logits for a
    group of continuations): these are copied.

    Outputs are allocated, not cleared: rows of q (and out, dq, ...) or of k that belong to no sequence, in front of cu[0] or behind cu[-1], are left as the
    allocator gave them, NaN included.  With arrays that are longer than their sequences cut the results, or clear these rows, before a product sums over all.

    Attention and decoding take products in bf16 with fp32 sums: the probabilities (and the gradients dS) are rounded to bf16 before the second product, see nat.h."""

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
