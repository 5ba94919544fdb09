"""How exact the weights of cross attention are on the GPU: rows that fit one or two blocks of 16 columns of a KV head hold them as a decode step does."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from tests import test_paged_precision as R
from tests.test_gpu_paged import F, bf16, ctx, cu_of, i32  # noqa: F401

pytestmark = pytest.mark.gpu

RUNS = [
    # rows, keys, hq, hkv, d
    ([5] * 16, [1500] * 16, 8, 8, 64),                       # beams over the states of their request
    ([2, 4, 1, 0, 3], [300, 4000, 129, 50, 777], 8, 2, 128),
    ([6], [2001], 20, 4, 64),                                # two blocks of columns
    ([1, 1], [900, 64], 28, 4, 128),                         # one row each, with prefix sums
    ([4] * 70, [65 + 3 * i for i in range(70)], 8, 4, 64),   # more sequences than a launch has
    ([2], [20000], 16, 1, 128),                              # keys of one tile in many parts
]


@pytest.mark.parametrize("case", RUNS, ids=[str(i) for i in range(len(RUNS))])
def test_weights_of_short_runs(F, ctx, case):
    """fp32 outputs: two terms of a weight (2-norm limits: see test_paged_precision, one term leaves 1.2e-3).  bf16 outputs are those, rounded once, but
    where what two terms leave (2^-16 of steps of 2^-8) brings one over the border, and near zero."""
    new, keys, hq, hkv, d = case
    rng = np.random.default_rng(sum(keys))
    q, qx = bf16(rng.normal(size=(sum(new), hq, d)))
    k, kx = bf16(rng.normal(size=(len(keys), hkv, max(keys), d)))
    v, vx = bf16(rng.normal(size=(len(keys), hkv, max(keys), d)))
    outs = []
    for fp32 in (1, 0):
        out = torch.empty(sum(new), hq, d, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
        F.flux_attn_cross(ctx, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, fp32), q, cu_of(new), max(new), max(keys), F.KVCache(k, v, i32(keys)), out)
        outs.append(out.double().cpu().numpy())
    ref, at = np.zeros(outs[0].shape), 0
    for b, (n, m) in enumerate(zip(new, keys)):
        ref[at:at + n] = S.cross(qx[at:at + n], kx[b, :, :m].transpose(1, 0, 2), vx[b, :, :m].transpose(1, 0, 2), 1 / np.sqrt(d))[0]
        at += n
    assert R.rel(outs[0], ref) <= R.TWO_TERMS, R.rel(outs[0], ref)
    assert R.rel(outs[1], outs[0]) <= R.ONE_TERM             # a rounding to bf16
    assert (outs[1] != R.to_bf16(outs[0])).mean() <= 0.02
    assert F.flux_last_device_status(ctx) == 0
