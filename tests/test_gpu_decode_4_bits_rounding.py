"""Attention of one token over the cache in 4 bits rounds to bf16 once: what it returns."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import attention as oattn
from oracle import kv_cache as okv

pytestmark = pytest.mark.gpu
U = 2.0 ** -8                   # half a step of bf16


@pytest.mark.parametrize("hq,hkv,D,page", [(4, 4, 64, 16), (28, 4, 128, 64), (16, 1, 128, 32), (8, 2, 64, 128)])
@pytest.mark.parametrize("spread", [0.3, 1.0, 4.0])
def test_one_rounding(hq, hkv, D, page, spread):
    """Limit: the result's rounding, U |out|; of sum_j P_j |v_j| the share R = 1e-5 (1 + max |S|) of scores, exponentials and sums in fp32, as the oracle has it, and U^2 = 2^-16 of the probabilities,
    which are taken as two numbers of 8 bits each."""
    from paper_2603_06619_amd.rollout import PagedCache, RolloutStage
    stage = RolloutStage(DEV)
    lens = [1, 2, 3, 17, 0, 40, 64, 333, 2500, 5000]
    width = -(-max(lens) // page)
    n_pages = len(lens) * width
    g = torch.Generator(device=DEV).manual_seed(hq + D)
    cache = PagedCache.empty(n_pages, hkv, page, D, device=DEV, fp4=True)
    new = lambda *s: torch.randn(s, generator=g, device=DEV)
    stage.write_cache(cache, new(n_pages * page, hkv, D).bfloat16(), (new(n_pages * page, hkv, D) * torch.exp(new(n_pages * page, hkv, 1))).bfloat16(),
                      torch.arange(n_pages * page, device=DEV))
    table = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32).view(len(lens), width)
    q = (spread * new(len(lens), hq, D)).bfloat16()
    out, lse = stage.decode(q, cache, table, torch.tensor(lens, dtype=torch.int32, device=DEV))
    k, v = (okv.group_values(getattr(cache, n).cpu().numpy(), getattr(cache, n + "_exp").cpu().numpy()) for n in ("k", "v"))
    args = (q.double().cpu().numpy(), k)
    ref = oattn.decode(*args, v, table.cpu().numpy(), np.array(lens), bounds=True)
    size = oattn.decode(*args, np.abs(v), table.cpu().numpy(), np.array(lens))["out"]                # sum_j P_j |v_j|
    limit = U * np.abs(ref["out"]) + (ref["e_lse"][..., None] + U * U) * 1.02 * size
    assert np.all(np.abs(out.double().cpu().numpy() - ref["out"]) <= limit)
