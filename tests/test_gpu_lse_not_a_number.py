"""A row whose scores are NaN has out and lse NaN; -inf is the lse of rows that see nothing, alone."""
import pytest
import torch

from nat_testlib import DEV
from test_gpu_attention import make, run, stage  # noqa: F401 (stage is a fixture)
from test_gpu_attention_split import key_parts
from test_gpu_kv_cache import decode_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens_q,lens_k,at", [([200, 30], [200, 30], 150), ([200, 30], [200, 30], 0), ([20], [3000], 7), ([90], [30], 75)])
def test_attention(stage, D, lens_q, lens_k, at):  # noqa: F811
    c = make(31, lens_q, lens_k, 4, 2, D)
    assert (key_parts(c) > 1) == (lens_k == [3000])
    want = run(stage, c, backward=False)
    unseen = lens_q[0] - lens_k[0]                                 # rows in front of the first that sees a key
    assert bool(want["lse"][:, :max(unseen, 0)].isneginf().all()) and bool(torch.isfinite(want["lse"][:, max(unseen, 0):]).all())
    c["q"][at, :, 0] = float("nan")
    got = run(stage, c, backward=False)
    assert bool(got["lse"][:, at].isnan().all()) and bool(got["out"][at].isnan().all())
    got["lse"][:, at], got["out"][at] = want["lse"][:, at], want["out"][at]
    assert torch.equal(got["lse"], want["lse"]) and torch.equal(got["out"], want["out"])
    if unseen > 0:                                                 # a query that sees nothing: whatever it holds
        c["q"][at] = 0.0
        want = run(stage, c, backward=False)
        c["q"][unseen - 1] = float("nan")
        got = run(stage, c, backward=False)
        assert torch.equal(got["lse"], want["lse"]) and torch.equal(got["out"], want["out"])


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("lens", [[40, 7, 0], [5000, 300, 0]])       # one workgroup per sequence and key head, and several
def test_decoding(stage, fp8, lens):  # noqa: F811
    c = decode_case(32, lens, 4, 2, 64, 32, fp8)
    want = stage.decode(c["q"], c["cache"], c["table"], c["lens"])
    assert bool(torch.isfinite(want[1][:2]).all()) and bool(want[1][2].isneginf().all())
    c["q"][1, 1:3] = float("nan")
    c["q"][2] = float("nan")
    out, lse = stage.decode(c["q"], c["cache"], c["table"], c["lens"])
    assert bool(lse[1, 1:3].isnan().all()) and bool(out[1, 1:3].isnan().all())
    out[1, 1:3], lse[1, 1:3] = want[0][1, 1:3], want[1][1, 1:3]
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
