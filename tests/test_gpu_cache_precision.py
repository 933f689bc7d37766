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


def far_below(fmt, n, scale_exponent, code, first_exponent=-4, units=27, hkv=1):
    """A first token whose probability is 2^units times that of every other one; behind its block, values of one code
    under one scale.  Every other dimension of the first block's values is 0."""
    d, blocks = 16, -(-n // 64)
    c = orc.Cache(fmt, blocks + 1, hkv, d, [np.random.default_rng(71).permutation(blocks + 1)[:blocks]], 1)
    c.k_scale[:], c.v_scale[:], c.weight[:] = 1, np.float32(2.0 ** scale_exponent), 0
    c.v[:] = code
    first = int(c.table[0, 0])
    c.v[first] = orc.encode(np.random.default_rng(72).uniform(-100, 100, (hkv, d, 64)) * (np.arange(d) % 2)[:, None], fmt)
    c.v_scale[first] = np.float32(2.0 ** first_exponent)
    c.k[first, :, 0, 0] = orc.encode(1.0, fmt)
    q = np.zeros((1, 2 * hkv, 1, d))
    q[:, :, :, 0] = units * np.log(2.0)
    return c, [n], q


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale_exponent,code,first,units", [
    (-100, 0, -4, 27), (-100, 1, -4, 27), (-90, 3, -4, 27), (-59, 3, -4, 27), (0, 0, -4, 27), (70, 1, -4, 27),
    (-100, 90, -100, 27), (-100, 90, -100, 36), (-95, 90, -95, 36), (61, 90, 61, 36)])
def test_tokens_count_whatever_the_size_of_their_values(fmt, dtype, scale_exponent, code, first, units):
    """Half a million tokens far below the first one: at 2^-27 they have 2^-8 of the sum between them, and every other
    dimension of the output is theirs alone."""
    c, lens, q = far_below(fmt, (1 << 19) - 5, scale_exponent, code, first, units)
    q = rounded(q, dtype)
    out, lse, got, mean_abs, largest = orc.attend(c, 0, q, lens, 1.0)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    for weights in (True, False):
        mine, mine_lse, gathered = call_attend(c, q, lens, dtype, scale=1.0, weights=weights)
        print("lse", mine_lse.ravel(), lse.ravel(), "largest share of the bound", (np.abs(mine - out) / tol).max(), flush=True)
        assert (np.abs(mine_lse - lse) <= tol_lse).all()
        assert (np.abs(mine - out) <= tol).all()
        if weights:
            # the first token's own weight: the sum's relative error and its rounding
            assert abs(gathered[c.table[0, 0], 0, 0] - got[0, 0][0]) <= got[0, 0][0] * (2 * tol_lse.max() + 2.0 ** -23)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scale_exponent,units", [(-100, 20), (-100, 27), (-100, 29), (-95, 32), (-90, 37), (-64, 37), (70, 34)])
def test_small_values_keep_the_bits_of_their_probabilities(fmt, scale_exponent, units):
    """p * scale about and below the least normal number, in dimensions that are the small tokens' alone; heads enough for
    a wave to have several blocks, so that three of sixteen are behind the large token."""
    c, lens, q = far_below(fmt, 1024, scale_exponent, 90, scale_exponent, units, 128)
    q = rounded(q, "f32")
    out, lse, got, mean_abs, largest = orc.attend(c, 0, q, lens, 1.0)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, "f32", dims=1)
    codes = np.abs(c.tokens(0, 0, 1024)[1]).sum(axis=0) * 2.0 ** -scale_exponent
    tol += codes * 2.0 ** -133                        # below the normal numbers p * scale is whole steps of bf16's least one
    for weights in (False, True):
        mine, mine_lse, gathered = call_attend(c, q, lens, "f32", scale=1.0, weights=weights)
        print("largest share of the bound", (np.abs(mine - out) / tol).max(), flush=True)
        assert (np.abs(mine - out) <= tol).all() and (np.abs(mine_lse - lse) <= tol_lse).all()


def many_tokens(n=(1 << 20) + 17, end=112):
    """A row whose values differ from one stretch of 36 blocks to the next, and whose last 17 tokens (codes of `end`) have a
    fiftieth of the probability between them: a missing block, stretch or end shows."""
    rng = np.random.default_rng(73)
    d, blocks = 16, -(-n // 64)
    c = orc.Cache(orc.INT8, blocks + 3, 1, d, [rng.permutation(blocks + 3)[:blocks]], 1)
    c.k_scale[:], c.v_scale[:] = 2.0 ** -5, 2.0 ** -6
    c.weight[:] = rng.random(c.weight.shape, dtype=np.float32) ** 4
    at = c.table[0]
    c.k[at] = rng.integers(-8, 9, (blocks, 1, 64, d)).astype(np.int8).view(np.uint8)
    mean = rng.integers(-90, 91, (-(-blocks // 36), 1, d, 1))[np.arange(blocks) // 36]
    c.v[at] = (mean + rng.integers(-20, 21, (blocks, 1, d, 64))).astype(np.int8).view(np.uint8)
    c.k[at[-1], 0, :17, 0] = end
    q = rng.standard_normal((1, 2, 1, d)) * 0.5
    q[..., 0] = 2
    return c, [n], q


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", [False, True])
def test_every_block_of_a_million_tokens(dtype, weights):
    c, lens, q = many_tokens()
    q = rounded(q, dtype)
    out, lse, got, mean_abs, largest = orc.attend(c, 0, q, lens, 1.0)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    mine, mine_lse, gathered = call_attend(c, q, lens, dtype, scale=1.0, weights=weights)
    print("largest share of the bounds", (np.abs(mine - out) / tol).max(), (np.abs(mine_lse - lse) / tol_lse).max(), flush=True)
    assert (np.abs(mine - out) <= tol).all()
    assert (np.abs(mine_lse - lse) <= tol_lse).all()
    if weights:
        n, at = lens[0], c.table[0]
        want = c.weight[at, 0].astype(np.float64).ravel()[:n] + got[0, 0]
        mine = gathered[at, 0].ravel()
        # a probability is as far off as its logit and the log-sum-exp; then the sum over the heads, and with the old weight
        assert (np.abs(mine[:n] - want) <= got[0, 0] * (2 * tol_lse.max() + 2.0 ** -22) + want * 2.0 ** -23).all()
        assert (mine[n:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens,hkv,group,window,d", [([1500, 300], 2, 2, 2, 64), ([900, 64, 65], 4, 8, 4, 128), ([700] * 3, 1, 5, 1, 80),
                                                     ([400] * 40, 8, 4, 1, 32), ([2100, 63], 2, 1, 40, 256)])
def test_ordinary_rows(fmt, dtype, lens, hkv, group, window, d):
    rng = np.random.default_rng([75, d, fmt])
    c = random_cache(rng, fmt, lens, hkv, d, 1)
    q = rounded(rng.standard_normal((len(lens), hkv * group, window, d)), dtype)
    out, lse, _, mean_abs, largest = orc.attend(c, 0, q, lens, d ** -0.5, causal=window > 1)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    for weights in (False, True):
        mine, mine_lse, _ = call_attend(c, q, lens, dtype, causal=int(window > 1), weights=weights)
        print("largest share of the bounds", (np.abs(mine - out) / tol).max(), flush=True)
        assert (np.abs(mine - out) <= tol).all() and (np.abs(mine_lse - lse) <= tol_lse).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,d,group,window", [(orc.E4M3, 144, 16, 1), (orc.INT8, 160, 5, 3), (orc.E4M3, 176, 4, 4), (orc.E4M3, 128, 8, 4),
                                                (orc.INT8, 80, 17, 1)])
def test_weights_with_all_of_lds(fmt, d, group, window):
    """Whole rows whose logits fill what LDS the waves' outputs and the queries leave, and go on in the workspace."""
    rng = np.random.default_rng([76, d])
    lens = [int(x) for x in rng.integers(0, 200, 32)]
    lens[7], lens[31] = 2100, 2000
    c = random_cache(rng, fmt, lens, 8, d, 1)
    q = rounded(rng.standard_normal((32, 8 * group, window, d)), "bf16")
    out, lse, got, mean_abs, largest = orc.attend(c, 0, q, lens, d ** -0.5, causal=window > 1)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, "bf16")
    mine, mine_lse, gathered = call_attend(c, q, lens, "bf16", causal=int(window > 1))
    fine = np.isfinite(lse)
    assert (np.isneginf(mine_lse) == ~fine).all() and (np.abs(mine - out) <= tol).all()
    assert (np.abs(mine_lse[fine] - lse[fine]) <= tol_lse[fine]).all()
    for (row, hh), x in got.items():
        at = c.table[row, :-(-len(x) // 64)]
        want = c.weight[at, hh].astype(np.float64).ravel()[:len(x)] + x
        error = np.abs(gathered[at, hh].ravel()[:len(x)] - want)
        # every probability is as far off as its logit and the log-sum-exp, and one sum of up to 32 of them
        assert (error <= x * (2 * tol_lse[fine].max() + 40 * 2.0 ** -23) + want * 2.0 ** -23 + 1e-37).all()
