"""flux_attn_prefill_paged computes the first max_q_len query rows of a sequence and leaves the others as they were, whatever tiles
the rows share and however their pages are shared out."""
import pytest
import torch

from tests.test_gpu_paged import FA, SA, F, attention_case, ctx, cu_of, tolerance  # noqa: F401
from tests.test_gpu_paged_prefill import check, prefill_ref

pytestmark = pytest.mark.gpu

CASES = [
    # new rows, cached before them, max_q_len, hq, hkv, d
    ([60, 60], [0, 30], 10, 8, 2, 128),                      # 40 rows of a tile of 64
    ([60, 5, 60], [0, 0, 30], 10, 7, 1, 128),                # group 7: 70 rows of a tile of 128, the last token behind the bound in part
    ([70], [0], 33, 4, 4, 64),                               # one head a tile: 33 rows, and 66 with the bound of the next case
    ([70], [0], 66, 4, 4, 64),                               # two tiles, of which the second ends in the bound
    ([300, 2, 100], [40, 700, 0], 50, 14, 2, 64),
    ([60, 60], [7000, 3000], 20, 8, 2, 128),                 # pages shared out, rows merged
    ([40], [5000], 19, 7, 1, 64),
    ([3, 9], [9000, 40], 2, 16, 1, 128),                     # runs, worked on like decode calls
]


@pytest.mark.parametrize("fp32", [1, 0])
@pytest.mark.parametrize("mode", [FA, SA])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_rows_beyond_the_bound_are_left_as_they_were(F, ctx, case, mode, fp32):
    rows, past, most, hq, hkv, d = case
    lens = [a + b for a, b in zip(rows, past)]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=sum(lens) + most, rows=rows)
    out = torch.full((sum(rows), hq, d), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, 20, 500, 0.0, fp32)
    modes = torch.full((len(rows),), mode, dtype=torch.uint8, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), most, max(lens), kv, pt, modes, out)
    ref = prefill_ref(qf, seqs, rows, [mode] * len(rows), 20, 500)
    asked, at = [], 0
    for n in rows:
        asked += range(at, at + min(n, most))
        at += n
    left = [i for i in range(at) if i not in set(asked)]
    check(out[asked], ref[asked], tolerance(qf, seqs, d), seqs)
    assert (out[left] == 7).all()
    assert F.flux_last_device_status(ctx) == 0
