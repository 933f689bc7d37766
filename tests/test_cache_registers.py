"""Registers of the built cache kernels: the forms that large caches are read, filled and pruned with spill nothing, and
the attention's keep two waves on every SIMD."""
import re

from test_kernel_registers import _fits, kernels  # noqa: F401  (the fixture)


def test_attention_of_up_to_sixteen_rows(kernels):  # noqa: F811
    seen = 0
    for name, k in kernels.items():
        m = re.search(r"attend_split<[01], unsigned short, ([12]), (true|false), 1, true>", name)
        if m:
            assert _fits(k, 3 if m.group(1) == "1" else 2), name
            seen += 1
    assert seen == 2 * 2 * 2


def test_fill_and_evict(kernels):  # noqa: F811
    found = [k for name, k in kernels.items() if "evict_move<" in name or re.search(r"cache_fill<[01], unsigned short, [24]>", name)]
    assert len(found) == 4 + 4 and all(_fits(k, 4) for k in found)
