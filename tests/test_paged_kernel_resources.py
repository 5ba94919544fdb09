"""What the host and the device code assume about the compiled kernels of the paged cache (registers and LDS; no GPU needed)."""
import os
import re

from tests.test_kernel_resources import kernels, workgroups_per_cu  # noqa: F401

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_07394_amd", "csrc")


def test_decode_calls_run_side_by_side(kernels):
    """Up to 512 workgroups, two per CU; of eight waves, and runs of two blocks of columns at head dimension 128, up to 256, one per CU.
    A part waits for no other, so this is speed, not safety; no instance may keep vector registers in memory."""
    assert int(re.search(r"kPagedFewWgs = (\d+);", open(os.path.join(CSRC, "paged.h")).read()).group(1)) == 256
    names = [n for n in kernels if "paged_decode_kernel" in n]
    assert len(names) == 28
    for n in names:
        d, waves, qb = (int(x) for x in re.search(r"ILi(\d+)ELb[01]ELi(\d)ELb[01]ELi(\d)E", n).groups())
        most = 256 if (d, qb) == (128, 2) or waves == 8 else 512
        assert kernels[n]["max_flat_workgroup_size"] == 64 * waves
        assert 256 * workgroups_per_cu(kernels[n]) >= most, (n, kernels[n])
        assert kernels[n]["vgpr_spill_count"] == 0, n


def test_prefill_rules_count_on_workgroups_side_by_side(kernels):
    """paged_resident: per CU two at head dimension 128, three and (tiles of 64 rows) four at 64."""
    src = open(os.path.join(CSRC, "paged.h")).read()
    assert "return head_dim == 128 ? 2 : (bm == 64 ? 4 : 3);" in src
    names = [n for n in kernels if "paged_prompt_kernel" in n]
    assert len(names) == 4
    for n in names:
        d, qb = (int(x) for x in re.search(r"ILi(\d+)ELi(\d)E", n).groups())
        assert workgroups_per_cu(kernels[n]) >= (2 if d == 128 else 4 if qb == 1 else 3), (n, kernels[n])
        assert kernels[n]["vgpr_spill_count"] == 0, n


def test_the_other_kernels_spill_nothing(kernels):
    names = [n for n in kernels if any(k in n for k in ("page_plan", "page_release", "append_paged", "paged_prompt_merge"))]
    assert len(names) == 6
    for n in names:
        assert kernels[n]["vgpr_spill_count"] == 0 and kernels[n]["group_segment_fixed_size"] <= 163840, n
