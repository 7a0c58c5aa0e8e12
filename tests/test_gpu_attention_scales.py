"""The least and the largest scales: "> 0 and finite" is all that is asked of them."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from test_gpu_attention import check, host, make, run, stage  # noqa: F401 (stage is a fixture)
from test_gpu_kv_cache import check_decode, decode_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [1e-30, 2e-38, 1.2e-38, 1e-38])
@pytest.mark.parametrize("lens_q,lens_k", [([150, 3], [150, 3]), ([20], [3000])])
def test_vanishing_scores(stage, D, scale, lens_q, lens_k):  # noqa: F811
    """Scores of about 0: the mean of the values that a row sees, and the logarithm of their number."""
    c = make(41, lens_q, lens_k, 4, 2, D)
    check(c, run(stage, c, scale=scale, backward=False), scale=scale, names=("out", "lse"))


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("scale", [1e-30, 1.2e-38])
def test_vanishing_scores_in_decoding(stage, fp8, scale):  # noqa: F811
    c = decode_case(42, [40, 0, 5000], 4, 2, 64, 32, fp8)
    check_decode(c, *stage.decode(c["q"], c["cache"], c["table"], c["lens"], scale=scale), scale=scale)
