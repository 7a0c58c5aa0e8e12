"""Every array of a call that is on another device than the current one is refused, one by one: a kernel launched here cannot reach it."""
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu


class Elsewhere(torch.Tensor):
    """A tensor that says it is on another device."""

    def get_device(self):
        return 1

    @property
    def device(self):
        return torch.device("cuda", 1)


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def normal(*shape):
    return torch.randn(shape, device=DEV).bfloat16()


def embed():
    return dict(ids=ints(1, 0), E=normal(4, 16), scale=1.0, out=normal(2, 16))


def embed_bwd():
    import paper_2603_06619_amd as nat
    return dict(ids=ints(1, 0), dout=normal(2, 16), scale=1.0, dE=torch.zeros((4, 16), device=DEV), accumulate=False,
                workspace=torch.empty(nat.embed_bwd_workspace_bytes(2, 4, 16), dtype=torch.uint8, device=DEV))


def norm_rope():
    return dict(q=normal(2, 4, 64), k=normal(2, 2, 64), q_weight=normal(64), k_weight=normal(64), position_ids=ints(3, 4),
                inv_freq=torch.ones(32, dtype=torch.float64, device=DEV), eps=1e-6, interleaved=False, q_out=normal(2, 4, 64), k_out=normal(2, 2, 64))


def norm_rope_bwd():
    import paper_2603_06619_amd as nat
    args = {name: x for name, x in norm_rope().items() if name not in ("q_out", "k_out")}
    return dict(args, dq_out=normal(2, 4, 64), dk_out=normal(2, 2, 64), dq=normal(2, 4, 64), dk=normal(2, 2, 64), dq_weight=torch.zeros(64, device=DEV),
                dk_weight=torch.zeros(64, device=DEV), accumulate=False,
                workspace=torch.empty(nat.qk_norm_rope_bwd_workspace_bytes(2, 64), dtype=torch.uint8, device=DEV))


def state(change):
    return dict(block_table=ints(1, -1, 2, -1).view(2, 2), seq_lens=ints(3, 16), **{change: ints(1, 1)}, free_pages=ints(0, 3, 0, 0), counts=ints(2, 0), page_size=16)


def reserve():
    return dict(state("new_lens"), rows_cap=2, counts_out=ints(0, 0), seq_lens_out=ints(0, 0), start=ints(0, 0), cu_new=ints(0, 0, 0),
                slots=torch.zeros(2, dtype=torch.int64, device=DEV), position_ids=ints(0, 0), workspace=torch.empty(256, dtype=torch.uint8, device=DEV))


def release():
    return dict(state("keep_lens"), counts_out=ints(0, 0), seq_lens_out=ints(0, 0), workspace=torch.empty(256, dtype=torch.uint8, device=DEV))


def cache(**kind):
    from paper_2603_06619_amd.rollout import PagedCache
    c = PagedCache.empty(4, 2, 16, 64, device=DEV, **kind)
    for x in (c.k, c.v, c.k_exp, c.v_exp):
        if x is not None:
            x.view(torch.uint8).zero_()
    return c


def write(**kind):
    return dict(cache=cache(**kind), k=normal(2, 2, 64), v=normal(2, 2, 64), slots=torch.tensor([3, 40], device=DEV))


def read(**kind):
    return dict(cache=cache(**kind), block_table=ints(1, 0, 2, 3).view(2, 2), cu_k=ints(0, 5, 30), k=normal(30, 2, 64), v=normal(30, 2, 64))


def decode(**kind):
    import paper_2603_06619_amd as nat
    table = torch.arange(200, dtype=torch.int32, device=DEV).view(2, 100) % 4           # as long as needs a workspace
    need = nat.attn_decode_workspace_bytes(2, 4, 2, 64, 1600)
    assert need > 0
    return dict(cache=cache(**kind), q=normal(2, 4, 64), block_table=table, seq_lens=ints(20, 1600), scale=0.1, out=normal(2, 4, 64),
                lse=torch.zeros((2, 4), device=DEV), workspace=torch.empty(need, dtype=torch.uint8, device=DEV))


FORMATS = [dict(), dict(fp8=True), dict(fp4=True)]
CALLS = [("nat_embed", embed, {}), ("nat_embed_bwd", embed_bwd, {}), ("nat_qk_norm_rope", norm_rope, {}), ("nat_qk_norm_rope_bwd", norm_rope_bwd, {}),
         ("nat_kv_reserve", reserve, {}), ("nat_kv_release", release, {})] + \
        [(name, make, kind) for name, make in (("nat_kv_write", write), ("nat_kv_read", read), ("nat_attn_decode", decode)) for kind in FORMATS]


@pytest.mark.parametrize("name,make,kind", CALLS, ids=[f"{name}{'-'.join(['', *kind])}" for name, _, kind in CALLS])
def test_each_array(name, make, kind):
    import paper_2603_06619_amd as nat
    call, args = getattr(nat, name), make(**kind)
    call(**args)                                         # as they are, they are fine
    torch.cuda.synchronize()
    tried = 0
    for arg, x in args.items():
        if isinstance(x, nat.KvCache):
            arrays = [t for t in (x.k, x.v, x.k_exp, x.v_exp) if t is not None]
            for i in range(len(arrays)):
                with pytest.raises(ValueError, match="cuda:1"):
                    nat.KvCache(*(t.as_subclass(Elsewhere) if i == j else t for j, t in enumerate(arrays)))
            with pytest.raises(ValueError, match="current device"):
                call(**dict(args, **{arg: nat.KvCache(*(t.as_subclass(Elsewhere) for t in arrays))}))
            tried += 1
        elif isinstance(x, torch.Tensor):
            with pytest.raises(ValueError, match="current device"):
                call(**dict(args, **{arg: x.as_subclass(Elsewhere)}))
            tried += 1
    assert tried >= 3
    call(**args)
    torch.cuda.synchronize()
