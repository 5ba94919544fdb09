"""What the host and the device code of heads, page moves and cross attention assume about their kernels (registers and LDS; no GPU needed)."""
import os
import re

from tests.test_kernel_resources import kernels, workgroups_per_cu  # noqa: F401

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_07394_amd", "csrc")
KERNELS = {"head_rows_kernel": 4, "qkv_rows_kernel": 4, "qkv_quant_kernel": 4, "page_fork_kernel": 2, "page_fork_end_kernel": 1, "page_compact_kernel": 1,
           "page_renumber_kernel": 1, "page_copy_kernel": 2, "cross_tile_kernel": 4, "cross_run_kernel": 4, "cross_join_kernel": 8}


def test_no_vector_register_lives_in_memory(kernels):
    for name, count in KERNELS.items():
        names = [n for n in kernels if name in n]
        assert len(names) == count, names
        for n in names:
            assert kernels[n]["vgpr_spill_count"] == 0 and workgroups_per_cu(kernels[n]) >= 1, (n, kernels[n])


def test_cross_rules_count_on_workgroups_side_by_side(kernels):
    src = open(os.path.join(CSRC, "cross.h")).read()
    assert "return 256 * (head_dim == 128 ? 2 : 3); }" in src and "kCrossRunWgs = 512;" in src
    for n in [n for n in kernels if "cross_tile_kernel" in n or "cross_run_kernel" in n]:
        d = int(re.search(r"ILi(\d+)E", n).group(1))
        assert workgroups_per_cu(kernels[n]) >= (2 if d == 128 or "cross_run" in n else 3), (n, kernels[n])
