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


def test_no_form_of_any_cache_kernel_spills(kernels):  # noqa: F811
    """Every form, with the waves per SIMD that it is launched for (attend_waves)."""
    seen = dict.fromkeys(("attend_split", "attend_join", "evict_select", "evict_move", "cache_fill", "cache_append"), 0)
    for name, k in kernels.items():
        kind = re.search(r"\b(attend_split|attend_join|evict_select|evict_move|cache_fill|cache_append)<", name)
        if not kind:
            continue
        seen[kind.group(1)] += 1
        waves, m = 1, re.search(r"attend_split<[01], (float|unsigned short), ([1-4]), (?:true|false), ([12]), ", name)
        if m:
            nj, qt, bf16 = int(m.group(2)), int(m.group(3)), m.group(1) != "float"
            waves = (3 if (nj, qt) == (1, 1) else 2 if nj <= 3 else 1) if bf16 else 2 if nj <= 2 and qt == 1 else 1
        assert _fits(k, waves), name
    assert seen == {"attend_split": 2 * 2 * 16, "attend_join": 2, "evict_select": 4, "evict_move": 4, "cache_fill": 12,
                    "cache_append": 4}
