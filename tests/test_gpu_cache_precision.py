"""kvc_cache_attend within bounds that count its roundings: what is lost by fewer bits or by a missing token shows."""
import numpy as np
import pytest

from cache_testlib import attend_bounds, call_attend, random_cache, rounded
from oracle import cache_oracle as orc

FORMATS = [orc.E4M3, orc.INT8]


def few_tokens(fmt, d, group, window, hkv=2):
    """Short rows and small logits: probabilities alike and the roundings of each one in the outputs."""
    rng = np.random.default_rng([70, fmt, d, group, window])
    lens = [3, 7, 21, 45]
    c = random_cache(rng, fmt, lens, hkv, d, 1)
    return c, lens, rounded(rng.standard_normal((4, hkv * group, window, d)) * 0.2, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [16, 64, 96, 128, 192])
@pytest.mark.parametrize("group,window", [(1, 1), (4, 4), (17, 1), (5, 4), (4, 8), (9, 5)])   # 1 to 45 rows to a KV head
def test_probabilities_have_sixteen_bits(fmt, d, group, window):
    c, lens, q = few_tokens(fmt, d, group, window)
    out, lse, _, mean_abs, largest = orc.attend(c, 0, q, lens, d ** -0.5)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, "bf16")
    for weights in (False, True):
        mine, mine_lse, _ = call_attend(c, q, lens, "bf16", weights=weights)
        share = np.abs(mine - out) / tol
        print("largest share of the bound", share.max(), flush=True)
        assert (share <= 1).all()
        assert (np.abs(mine_lse - lse) <= tol_lse).all()
