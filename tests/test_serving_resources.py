"""The serving kernels keep their state in registers: no scratch memory, and two workgroups of the many-row attention to a
compute unit.  (The sampling kernel is left out: 128 registers a thread at 16 wavefronts, it keeps a row's parameters in scratch.)"""
import pytest

from tests.test_kernel_resources import load

KERNELS = {"paged_attn_kernel": ("kernels_paged_attn.hip", 16), "paged_attn_wide_kernel": ("kernels_paged_attn.hip", 4),
           "paged_attn_both_kernel": ("kernels_paged_attn.hip", 4), "paged_attn_f32_kernel": ("kernels_paged_attn.hip", 3),
           "paged_combine_kernel": ("kernels_paged_attn.hip", 4), "paged_append_kernel": ("kernels_paged_cache.hip", 10),
           "page_copy_kernel": ("kernels_paged_cache.hip", 4)}


@pytest.mark.parametrize("fragment", sorted(KERNELS))
def test_no_scratch_memory(fragment):
    src, count = KERNELS[fragment]
    found = {k: v for k, v in load(src).items() if fragment in k}
    assert len(found) == count, sorted(found)
    for name, res in found.items():
        assert res["ScratchSize"] == 0 and res["VGPRs Spill"] == 0, (name, res)
        if "wide" in name or "both" in name:
            assert res["Occupancy"] >= 2, (name, res)
