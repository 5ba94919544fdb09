"""Short runs of queries behind a cached context (drafted tokens) are worked on like decode calls, and their rows are as exact: a weight
is held to 2^-16, for fp32 outputs to 2^-24 (limits: tests/test_paged_precision.py)."""
import numpy as np
import pytest
import torch

from tests import helpers as H
from tests import test_paged_precision as R
from tests.test_gpu_paged import FA, SA, F, ctx, cu_of, tolerance  # noqa: F401
from tests.test_gpu_paged_precision import SINK, WINDOW, case_of

pytestmark = pytest.mark.gpu

CASES = [
    # new rows, cached before them, hq, hkv, d
    ([5, 8, 3], [2000, 700, 5000], 8, 2, 128),               # two blocks of columns
    ([4] * 12, [600 + 50 * i for i in range(12)], 16, 4, 64),
    ([2, 2], [900, 3000], 16, 1, 128),
    ([2, 0, 1], [900, 3, 3000], 14, 2, 128),                 # group 7
    ([1] * 5, [500, 64, 63, 2000, 130], 8, 2, 64),           # one query each
    ([1, 0, 1], [3000, 5, 600], 40, 2, 128),                 # groups of 20 and 32: the heads of one query take two blocks
    ([1], [900], 32, 1, 64),
]


@pytest.mark.parametrize("mode", [FA, SA])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_weights_of_drafted_tokens(F, ctx, case, mode):
    rows, past, hq, hkv, d = case
    lens, kv, pt, q, qf, seqs, ref, _ = case_of(F, rows, past, hq, hkv, d, mode, sum(past))
    cfgs = [F.attn_cfg(hq, hkv, d, SINK, WINDOW, 0.0, fp32) for fp32 in (0, 1)]
    modes = torch.full((len(rows),), mode, dtype=torch.uint8, device="cuda")
    v = max(float(np.abs(s[1]).max()) for s in seqs)
    for fp32 in (1, 0):
        out = torch.empty(sum(rows), hq, d, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
        F.flux_attn_prefill_paged(ctx, cfgs[fp32], q, cu_of(rows), max(rows), max(lens), kv, pt, modes, out)
        got = H.torch_to_f64(out)
        bound = tolerance(qf, seqs, d) * v                   # (with two terms)
        assert (np.abs(got - ref) <= (bound if fp32 else bound + 2.0 ** -8 * (np.abs(ref) + bound))).all()
        assert R.rel(got, ref) <= (R.THREE_TERMS if fp32 else R.ONE_TERM)   # (bf16: the rounding of the output)
        # the last rows are what a decode call gives for them, to the same limits
        last = [sum(rows[:b + 1]) - 1 for b in range(len(rows)) if rows[b]]
        one = torch.empty(len(rows), hq, d, dtype=out.dtype, device="cuda")
        F.flux_attn_decode_paged(ctx, cfgs[fp32], q[[max(0, sum(rows[:b + 1]) - 1) for b in range(len(rows))]].contiguous(), max(lens), kv, pt, modes, one)
        one = H.torch_to_f64(one)[[b for b in range(len(rows)) if rows[b]]]
        assert R.rel(got[last], one) <= (2 * R.THREE_TERMS if fp32 else R.ONE_TERM / 2)   # (few results lie so near a border that they are rounded apart)
    assert F.flux_last_device_status(ctx) == 0
