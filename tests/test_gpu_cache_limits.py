"""The block cache at its far ends: pools beyond 4 GiB, rows of a million tokens, the largest batch, many heads, calls that
run at once on two streams."""
import numpy as np
import pytest
import torch

import paper_2509_05165_amd as kv
from cache_testlib import POOLS, Device, dev, params, random_cache, stream, workspace
from oracle import cache_oracle as orc
from test_gpu_cache_attend import check

pytestmark = pytest.mark.gpu


class Far:
    """The blocks of a small cache at the far end of pools of `blocks` blocks, the rest of which nobody has written."""

    def __init__(self, c, blocks):
        self.c, self.shift, self.t = c, blocks - len(c.k), {}
        for n in POOLS:
            a = getattr(c, n)
            self.t[n] = torch.empty((blocks,) + a.shape[1:], dtype=torch.uint8 if a.dtype == np.uint8 else torch.float32, device="cuda")
            self.t[n][self.shift:] = dev(a)
        self.t["table"] = dev(self.table(c.table))
        self.struct = kv.KvcCache(c.fmt, blocks, c.table.shape[1], *[self.t[n].data_ptr() for n in POOLS + ("table",)])

    def table(self, table):
        return np.where((table >= 0) & (table < len(self.c.k)), table + self.shift, -1).astype(np.int32)

    def same(self, c):
        for n in POOLS:
            np.testing.assert_array_equal(self.t[n][self.shift:].cpu().numpy().view(np.uint8), np.ascontiguousarray(getattr(c, n)).view(np.uint8), err_msg=n)


def test_pools_beyond_32_bits():
    """70000 blocks of 8 heads of 128: codes, scales and weights at byte offsets beyond 2^32, 2^31 elements."""
    rng = np.random.default_rng(60)
    lens = [150, 64, 1, 300]
    c = random_cache(rng, orc.E4M3, lens, 8, 128, 2, spare=30)
    far = Far(c, 70000)
    assert far.t["k"].numel() > 1 << 32
    near = Device(c)
    k, v = (rng.standard_normal((2, 8, 3, 128)) * 4 for _ in "kv")
    tk, tv, t_len = dev(k, "bf16"), dev(v, "bf16"), dev(np.asarray(lens, np.int32))
    p = params(c, 2, 32, "bf16", window=3, causal_tail=1)
    need = kv.kvc_cache_attend_workspace(p, 320, True)
    q, outs = dev(rng.standard_normal((2, 32, 3, 128)), "bf16"), []
    for x in (near, far):
        ws, out = workspace(need), torch.empty_like(q)
        kv.kvc_cache_append(p, 1, tk.data_ptr(), tv.data_ptr(), t_len.data_ptr(), x.struct, stream())
        kv.kvc_cache_attend(p, 1, q.data_ptr(), t_len.data_ptr(), 320, x.struct, out.data_ptr(), ws.data_ptr(), need, stream(),
                            weight_in=x.t["weight"].data_ptr(), weight_out=x.t["weight"].data_ptr())
        outs.append(out)
    assert torch.equal(*outs)
    for n in POOLS:
        setattr(c, n, near.t[n].cpu().numpy())
    far.same(c)
    # eviction and fill into the spare blocks
    spare = np.setdiff1d(np.arange(len(c.k)), c.table[(c.table >= 0) & (c.table < len(c.k))])
    table, at = np.full(c.table.shape, -1, np.int32), 0
    for r, n in enumerate((2, 1, 1, 3)):
        table[r, :n] = spare[at:at + n]
        at += n
    keep = np.array([100, 50, 1, 170], np.int32)
    out_len, t_keep, ws = torch.empty(4, dtype=torch.int32, device="cuda"), dev(keep), workspace(kv.kvc_cache_evict_workspace(p, 170))
    t_table = dev(far.table(table))
    kv.kvc_cache_evict(p, t_len.data_ptr(), t_keep.data_ptr(), 170, far.struct, t_table.data_ptr(), out_len.data_ptr(), ws.data_ptr(),
                       ws.numel(), stream())
    np.testing.assert_array_equal(out_len.cpu().numpy(), orc.evict(c, lens, keep, table, 170))
    far.same(c)
    rows = torch.randn((2, 8, 300, 128), device="cuda").to(torch.bfloat16)
    offsets = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64))
    kv.kvc_cache_fill(params(c, 2, 32, "bf16", window=1), [x.data_ptr() for x in rows[:, :, :300]], [x.data_ptr() for x in rows], 0,
                      t_len.data_ptr(), offsets.data_ptr(), [0, 150, 300], sum(lens), far.struct, stream())
    x = rows.double().cpu().numpy()
    orc.fill(c, x, x, None, lens, [0, 150, 300])
    far.same(c)


@pytest.mark.parametrize("weights", ["none", "add"])
def test_a_million_tokens(weights):
    rng = np.random.default_rng(61)
    lens = [(1 << 20) + 17]
    check(rng, random_cache(rng, orc.INT8, lens, 1, 16, 1), lens, 2, weights=weights)


def test_the_largest_batch_and_many_heads():
    rng = np.random.default_rng(62)
    lens = [int(x) for x in rng.integers(0, 130, 256)]
    check(rng, random_cache(rng, orc.E4M3, lens, 1, 16, 1), lens, 3)
    lens = [70, 200]
    check(rng, random_cache(rng, orc.E4M3, lens, 256, 16, 1), lens, 256)


def test_two_streams_at_once():
    """Calls on caches, workspaces and streams of their own, many in flight on each."""
    rng = np.random.default_rng(63)
    sets = []
    for seed in range(2):
        lens = [3000, 500 + seed]
        c = random_cache(rng, orc.E4M3, lens, 8, 64, 1)
        p = params(c, 2, 16, "bf16")
        need = kv.kvc_cache_attend_workspace(p, 3000, True)
        q = dev(rng.standard_normal((2, 16, 1, 64)), "bf16")
        sets.append((c, p, need, q, dev(np.asarray(lens, np.int32))))

    def run(s, x, out, device, ws, times):
        c, p, need, q, t_len = x
        for _ in range(times):
            kv.kvc_cache_attend(p, 0, q.data_ptr(), t_len.data_ptr(), 3000, device.struct, out.data_ptr(), ws.data_ptr(), need, s,
                                weight_in=device.t["weight"].data_ptr(), weight_out=device.t["weight"].data_ptr())

    want = []
    for x in sets:
        out, device = torch.empty_like(x[3]), Device(x[0])
        run(stream(), x, out, device, workspace(x[2]), 20)
        want.append((out, device.t["weight"]))
    outs, devices, spaces = [torch.empty_like(x[3]) for x in sets], [Device(x[0]) for x in sets], [workspace(x[2]) for x in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in (0, 1):
            run(streams[i].cuda_stream, sets[i], outs[i], devices[i], spaces[i], 1)
    torch.cuda.synchronize()
    for i in (0, 1):
        assert torch.equal(outs[i], want[i][0])
        assert torch.equal(devices[i].t["weight"].view(torch.int32), want[i][1].view(torch.int32))
