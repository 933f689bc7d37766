"""kvc_cache_attend against the oracle in float64: outputs, log-sum-exps and gathered weights."""
import numpy as np
import pytest
import torch

import paper_2509_05165_amd as kv
from cache_testlib import DTYPES, Device, attend_tolerance, dev, params, random_cache, rounded, stream, workspace
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu
FORMATS = [orc.E4M3, orc.INT8]


def check(rng, c, lens, hq, dtype="bf16", window=1, causal=0, layer=0, scale=0.0, max_length=None, weights="add",
          q_size=1.0, offset=0):
    batch = len(lens) // (c.layers * (c.hkv if c.unstructured else 1))
    q = rounded(rng.standard_normal((batch, hq, window, c.d)) * q_size, dtype)
    device, esz = Device(c), DTYPES[dtype][0].itemsize
    flat = dev(np.concatenate([np.zeros(offset), q.ravel()]), dtype)
    lengths = dev(np.asarray(lens, np.int32))
    out = torch.full((offset + q.size,), 7.0, dtype=DTYPES[dtype][0], device="cuda")
    lse = torch.full((batch, hq, window), 7.0, device="cuda")
    w_out = torch.full(c.weight.shape, 7.0, device="cuda")
    p = params(c, batch, hq, dtype, window, causal_tail=causal, softmax_scale=scale)
    most = max(max(lens), 0) if max_length is None else max_length
    size = kv.kvc_cache_attend_workspace(p, most, weights != "none")
    ws = workspace(size)
    w_in = {"add": device.t["weight"].data_ptr(), "set": 0, "none": 0}[weights]
    kv.kvc_cache_attend(p, layer, flat.data_ptr() + offset * esz, lengths.data_ptr(), most, device.struct,
                        out.data_ptr() + offset * esz, ws.data_ptr(), size, stream(), lse=lse.data_ptr(), weight_in=w_in,
                        weight_out=w_out.data_ptr() if weights != "none" else 0)
    ref, ref_lse, got, mean_abs, largest = orc.attend(c, layer, q, lens, scale or c.d ** -0.5, bool(causal), most)
    mine = out[offset:].double().cpu().numpy().reshape(q.shape)
    assert (out[:offset] == 7).all()
    err, tol = np.abs(mine - ref), attend_tolerance(c, q, mean_abs, largest, ref, dtype)
    print("largest share of the tolerance", (err / tol).max() if err.size else 0, flush=True)
    defined = ~np.isnan(ref_lse)                      # rows that read slots nobody wrote have no value
    assert (err <= tol)[defined].all()
    lse = lse.double().cpu().numpy()
    np.testing.assert_array_equal(np.isneginf(lse)[defined], np.isneginf(ref_lse)[defined])
    fine = np.isfinite(ref_lse)
    # the logits' own error (attend_tolerance), and the logarithm's and the product's rounding
    rel = largest * 2.0 ** -24 * 1.4427 * (c.d + 10) + 2.0 ** -20 + np.abs(np.where(fine, ref_lse, 0)) * 2.0 ** -22
    rel = np.where(defined, rel, 0)
    assert (np.abs(lse[fine] - ref_lse[fine]) <= (rel + c.table.shape[1] * 64 * 2.0 ** -24)[fine]).all()
    if weights == "none":
        assert (w_out == 7).all()
    else:
        mine = w_out.cpu().numpy()
        want = np.full(c.weight.shape, 7.0)
        tol = np.zeros(c.weight.shape)
        for (row, hh), x in got.items():
            for j in range(-(-len(x) // 64)):
                i = c.block(row, j)
                if i is None:
                    continue
                part = x[j * 64:(j + 1) * 64]
                want[i, hh, :len(part)] = part + (c.weight[i, hh, :len(part)] if weights == "add" else 0)
                tol[i, hh, :len(part)] = part * 4 * rel.max() + np.abs(want[i, hh, :len(part)]) * 2.0 ** -22 + 1e-37
        assert ((np.abs(mine - want) <= tol) | np.isnan(want)).all()
    device.same(c)                                    # the cache itself is only read
    return out, lse, w_out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [16, 32, 64, 80, 96, 128, 144, 192, 256])
def test_head_sizes(fmt, dtype, d):
    rng = np.random.default_rng([10, d, fmt])
    check(rng, random_cache(rng, fmt, [130, 65], 2, d, 1), [130, 65], 6, dtype, 2, 1)


@pytest.mark.parametrize("hq,hkv,window", [(1, 1, 1), (7, 1, 1), (28, 4, 1), (8, 8, 1), (16, 1, 1), (17, 1, 1), (8, 2, 5),
                                           (40, 8, 7), (64, 1, 1), (4, 1, 33)])
@pytest.mark.parametrize("fmt,dtype", [(orc.E4M3, "bf16"), (orc.INT8, "f32"), (orc.INT8, "bf16")])
def test_query_layouts(fmt, dtype, hq, hkv, window):
    rng = np.random.default_rng([11, hq, window])
    check(rng, random_cache(rng, fmt, [150, 40], hkv, 64, 1), [150, 40], hq, dtype, window, int(window > 1))


@pytest.mark.parametrize("lens", [[1], [0], [63, 64, 65], [0, 1, 2, 300], [4000], [255, 256, 257, 258], [9000, 3]])
@pytest.mark.parametrize("weights", ["add", "set", "none"])
def test_lengths(lens, weights):
    rng = np.random.default_rng([12, len(lens)])
    check(rng, random_cache(rng, orc.E4M3, lens, 1, 32, 1), lens, 4, "bf16", weights=weights)


@pytest.mark.parametrize("causal", [0, 1])
def test_more_queries_than_tokens(causal):
    """Queries before the first token see nothing: zeros and minus infinity."""
    rng = np.random.default_rng(13)
    out, lse, _ = check(rng, random_cache(rng, orc.INT8, [3, 0, 70], 2, 48, 1), [3, 0, 70], 4, "bf16", 6, causal)
    assert np.isneginf(lse[1]).all() and np.isneginf(lse[0][:, :3]).all() == bool(causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_rows_split_over_workgroups(dtype):
    rng = np.random.default_rng(14)
    lens = [20000, 77, 4097]
    check(rng, random_cache(rng, orc.E4M3, lens, 1, 64, 1), lens, 3, dtype)


def test_bounds_and_blocks_that_are_not_there():
    """max_length inside a row and beyond the table; lengths no row can have; entries that name no block."""
    rng = np.random.default_rng(15)
    c = random_cache(rng, orc.E4M3, [400, 130, 64, 200], 2, 64, 1)
    c.table[0, 2] = -1
    c.table[3, :] = 1 << 20                           # nothing of this row is there
    full = c.table.shape[1] * 64
    for lens, most in (([400, 130, 64, 200], 100), ([400, 130, -9, 200], 1 << 28), ([2 ** 31 - 1, 130, 64, 200], full)):
        check(rng, c, lens, 4, max_length=most)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_first_block_of_the_pool_is_nobodys(dtype):
    """Block 0, which stands in for entries that name no block, holds NaN codes and NaN scales."""
    rng = np.random.default_rng(38)
    c = random_cache(rng, orc.E4M3, [300, 64], 2, 64, 1)
    spare = int(np.setdiff1d(np.arange(len(c.k)), np.concatenate([c.table[0, :5], c.table[1, :1]]))[-1])
    if (c.table == 0).any() and spare:
        for name in ("k", "v", "k_scale", "v_scale", "weight"):
            getattr(c, name)[spare] = getattr(c, name)[0]
        c.table[c.table == 0] = spare
    c.k[0] = c.v[0] = 0x7F
    c.k_scale[0] = c.v_scale[0] = np.nan
    c.table[0, 1] = -1
    c.table[1, 0] = 1 << 30                           # nothing of this row is there
    for weights in ("add", "none"):
        check(rng, c, [300, 64], 4, dtype, weights=weights)


def test_layers_and_heads_with_rows_of_their_own():
    rng = np.random.default_rng(16)
    lens = list(rng.integers(0, 200, 2 * 3 * 4))
    c = random_cache(rng, orc.INT8, lens, 4, 32, 3, unstructured=True)
    for layer in range(3):
        check(rng, c, lens, 8, layer=layer, window=2, causal=1)
    lens = list(rng.integers(0, 200, 2 * 3))
    c = random_cache(rng, orc.INT8, lens, 4, 32, 3)
    check(rng, c, lens, 8, layer=2)


@pytest.mark.parametrize("fmt", FORMATS)
def test_extreme_logits(fmt):
    """Sharp attention whose largest logits come late, early and beyond what exp holds; a given scale."""
    rng = np.random.default_rng(17)
    for size, scale in ((40.0, 0.0), (300.0, 0.3), (1e-3, 0.0)):
        c = random_cache(rng, fmt, [500], 2, 64, 1)
        for i, x in ((0, 1.0), (3, 8.0), (7, 64.0)):
            c.k_scale[c.table[0, i]] *= x
        check(rng, c, [500], 4, "f32", q_size=size, scale=scale)
        check(rng, c, [500], 4, "bf16", q_size=size, scale=scale)


def test_scales_at_their_ends():
    """Blocks of the least scale, values of 2^88, a softmax scale that no product with it survives."""
    rng = np.random.default_rng(35)
    for e, scale in ((-100, 0.0), (80, 0.0), (-100, 1e-30)):
        c = random_cache(rng, orc.INT8, [150, 0], 2, 32, 1)
        c.v_scale[c.table[0, 1]] = np.float32(2.0 ** e)
        c.k_scale[c.table[0, 0]] = np.float32(2.0 ** -100)
        check(rng, c, [150, 0], 4, "f32", window=2, causal=1, scale=scale)


def test_pointers_off_sixteen_bytes():
    rng = np.random.default_rng(18)
    for dtype in ("bf16", "f32"):
        check(rng, random_cache(rng, orc.E4M3, [100], 2, 80, 1), [100], 4, dtype, offset=3)


def test_weights_in_place_and_repeated():
    """weight_out may be the cache's own weights: two calls add the probabilities twice, with equal bits each time."""
    rng = np.random.default_rng(19)
    c = random_cache(rng, orc.E4M3, [700, 20], 2, 64, 1)
    q, lengths = dev(rng.standard_normal((2, 4, 1, 64)), "bf16"), dev(np.array([700, 20], np.int32))
    p = params(c, 2, 4, "bf16")
    size = kv.kvc_cache_attend_workspace(p, 700, True)
    runs = []
    for _ in range(2):
        device, ws, out = Device(c), workspace(size), torch.empty_like(q)
        for _ in range(2):
            kv.kvc_cache_attend(p, 0, q.data_ptr(), lengths.data_ptr(), 700, device.struct, out.data_ptr(), ws.data_ptr(), size,
                                stream(), weight_in=device.t["weight"].data_ptr(), weight_out=device.t["weight"].data_ptr())
        runs.append(device.t["weight"].cpu().numpy())
    np.testing.assert_array_equal(runs[0].view(np.uint32), runs[1].view(np.uint32))
    gained = sum(float(np.nansum(runs[0][c.table[b, :n]] - c.weight[c.table[b, :n]])) for b, n in ((0, 11), (1, 1)))
    assert abs(gained - 2 * 2 * 4) < 1e-3              # two calls, two sequences, four heads


@pytest.mark.parametrize("seed", range(40))
def test_random_calls(seed):
    rng = np.random.default_rng([33, seed])
    layers, hkv, d = int(rng.integers(1, 3)), int(rng.integers(1, 4)), 16 * int(rng.integers(1, 17))
    unstructured, window = bool(rng.integers(0, 2)), int(rng.choice([1, 1, 2, 5, 9]))
    rows = int(rng.integers(1, 4)) * layers * (hkv if unstructured else 1)
    lens = [int(x) for x in rng.integers(0, int(rng.choice([70, 300, 2000])), rows)]
    c = random_cache(rng, int(rng.integers(0, 2)), lens, hkv, d, layers, unstructured=unstructured)
    check(rng, c, lens, hkv * int(rng.integers(1, 9)), str(rng.choice(["bf16", "f32"])), window, int(rng.integers(0, 2)),
          layer=int(rng.integers(0, layers)), weights=str(rng.choice(["add", "set", "none"])), q_size=float(rng.choice([0.3, 1, 4])))


@pytest.mark.parametrize("group,window,longest,weights", [(1, 1, 16384, "add"), (4, 1, 14001, "add"), (3, 8, 3001, "set"), (40, 1, 2500, "add"),
                                                          (2, 1, 16385, "add")])
def test_weights_of_long_whole_rows(group, window, longest, weights):
    """More than 64 blocks to a workgroup; logits that LDS holds, that it holds in part, and rows that are split after all."""
    rng = np.random.default_rng([37, group])
    lens = [int(x) for x in rng.integers(0, 300, 32)]
    lens[3], lens[30] = longest, longest // 2 + 1
    c = random_cache(rng, orc.E4M3, lens, 8, 16, 1)
    c.table[3, [1, -2 - (longest % 64 == 0)]] = -1
    check(rng, c, lens, 8 * group, window=window, causal=int(window > 1), weights=weights)


@pytest.mark.parametrize("batch,hkv,lens", [(64, 8, (1, 300)), (70, 8, (4000, 4400)), (20, 8, (1, 3000)), (9, 8, (500, 2500))])
def test_many_heads(batch, hkv, lens):
    """Every way in which a call is split over workgroups: whole rows, 64, 16 and 8 blocks at a time."""
    rng = np.random.default_rng([34, batch])
    lens = [int(x) for x in rng.integers(lens[0], lens[1], batch)]
    check(rng, random_cache(rng, orc.E4M3, lens, hkv, 16, 1), lens, 2 * hkv)


@pytest.mark.parametrize("group,window,weights", [(1, 1, "add"), (4, 1, "set"), (8, 1, "add"), (9, 1, "add"), (3, 3, "set"), (20, 1, "add")])
def test_weights_of_whole_rows(group, window, weights):
    """Heads enough for whole rows: logits in LDS (up to 126 KB of them and no longer), holes in the table."""
    rng = np.random.default_rng([36, group, window])
    lens = [int(x) for x in rng.integers(0, 1500, 63)] + [4096 if group <= 9 else 1500]
    c = random_cache(rng, orc.INT8, lens, 8, 16, 1)
    c.table[5, 1] = -1
    check(rng, c, lens, 8 * group, window=window, causal=int(window > 1), weights=weights)
