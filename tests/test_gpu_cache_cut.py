"""kvc_cache_evict down to few tokens of long rows: what stays, bit for bit, and that the blocks between are not read."""
import numpy as np
import pytest
import torch

import paper_2509_05165_amd as kv
from cache_testlib import dev, random_cache, stream, workspace
from oracle import cache_oracle as orc
from test_gpu_cache_evict import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8])
@pytest.mark.parametrize("n,keep,first,last", [(9000, 64, 4, 60), (9000, 64, 60, 4), (9001, 65, 1, 63), (9000, 7, 3, 4), (700, 64, 32, 32),
                                               (9000, 130, 4, 4)])
def test_both_ends_of_a_row(fmt, n, keep, first, last):
    rng = np.random.default_rng([100, n, keep, fmt])
    check(rng, random_cache(rng, fmt, [n, 130], 2, 80, 1), [n, 130], [keep, keep], first=first, last=last)


@pytest.mark.parametrize("seed", range(12))
def test_tokens_in_runs_and_alone(seed):
    """Target blocks whose tokens lie in one source block, in neighbours, in blocks far apart, at every slot."""
    rng = np.random.default_rng([101, seed])
    n = int(rng.integers(500, 6000))
    c = random_cache(rng, int(rng.integers(0, 2)), [n], 2, int(rng.choice([16, 64, 128, 208])), 1)
    c.weight[:] *= 0.1
    for h in range(2):
        for _ in range(int(rng.integers(1, 30))):
            at, run = int(rng.integers(0, n)), int(rng.choice([1, 1, 2, 5, 64, 200]))
            for t in range(at, min(n, at + run)):
                c.weight[c.table[0, t // 64], h, t % 64] += 1
    check(rng, c, [n], [int(rng.integers(1, 200))], first=int(rng.integers(0, 3)), last=int(rng.integers(0, 40)))


def test_blocks_without_a_kept_token_are_not_read():
    """64 tokens at the two ends of 131072 take about the time of the 64 at one end: the values' kernel needs two source
    blocks a head for both.  (The 2046 between, one after the other, would be a hundred times that.)"""
    n, hkv, d, width = 131072, 8, 128, 2048
    k = torch.zeros((width + 1, hkv, 64, d), dtype=torch.uint8, device="cuda")
    v = torch.zeros((width + 1, hkv, d, 64), dtype=torch.uint8, device="cuda")
    scales, weight = torch.ones((2, width + 1, hkv), device="cuda"), torch.zeros((width + 1, hkv, 64), device="cuda")
    table = dev(np.arange(width, dtype=np.int32)[None])
    target = torch.full_like(table, width)
    cache = kv.KvcCache(kv.KVC_INT8, width + 1, width, k.data_ptr(), v.data_ptr(), scales[0].data_ptr(), scales[1].data_ptr(),
                        weight.data_ptr(), table.data_ptr())
    lengths, keep = dev(np.array([n], np.int32)), dev(np.array([64], np.int32))
    out = torch.empty_like(lengths)
    times = []
    for first, last in ((0, 64), (4, 60)):
        p = kv.KvcParams(1, 1, hkv, hkv, d, 1, kv.KVC_BF16, keep_first=first, keep_last=last)
        ws = workspace(kv.kvc_cache_evict_workspace(p, 64))

        def call():
            kv.kvc_cache_evict(p, lengths.data_ptr(), keep.data_ptr(), 64, cache, target.data_ptr(), out.data_ptr(), ws.data_ptr(),
                               ws.numel(), stream())

        call()
        kv.kvc_profile_collect()
        kv.kvc_profile_enable(True)
        try:
            for _ in range(10):
                call()
            torch.cuda.synchronize()
        finally:
            kv.kvc_profile_enable(False)
        launches, ms = kv.kvc_profile_collect()["evict_move<v>"]
        times.append(ms / launches * 1e3)
    print("us of one end, of two", times, flush=True)
    assert times[1] < 10 * times[0]
