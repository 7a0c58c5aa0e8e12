"""The oracle's rows of NaN scores: NaN in out and lse, and -inf in lse for rows that see nothing, alone."""
import numpy as np

from oracle import attention as oattn


def test_rows_of_nan_scores():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 2, 8)), rng.standard_normal((3, 1, 8)), rng.standard_normal((3, 1, 8))
    good = oattn.attention(q, k, v, [0, 5], [0, 3])
    assert np.isneginf(good["lse"][:, :2]).all() and np.isfinite(good["lse"][:, 2:]).all()
    q[3, 0, 2] = np.nan
    q[0] = np.nan                                          # sees nothing
    r = oattn.attention(q, k, v, [0, 5], [0, 3])
    assert np.isnan(r["lse"][0, 3]) and np.isnan(r["out"][3, 0]).all()
    r["lse"][0, 3], r["out"][3, 0] = good["lse"][0, 3], good["out"][3, 0]
    assert np.array_equal(r["lse"], good["lse"]) and np.array_equal(r["out"], good["out"])
