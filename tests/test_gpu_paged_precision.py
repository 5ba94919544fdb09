"""What the paged attention kernels keep of weights and values, against float64, with the limits of tests/test_paged_precision.py: decode
holds a weight to 2^-16 (fp32 outputs 2^-24), the tiles of prefill to 2^-8, and neither rounds keys or values."""
import numpy as np
import pytest
import torch

from tests import helpers as H
from tests import test_paged_precision as R
from tests.test_gpu_paged import FA, SA, F, attention_case, ctx, cu_of, tolerance  # noqa: F401

pytestmark = pytest.mark.gpu

SINK, WINDOW = 20, 300


def case_of(F, rows, past, hq, hkv, d, mode, seed):
    lens = [a + b for a, b in zip(rows, past)]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=seed, rows=rows)
    refs, at = [], 0
    for n, length, (k, v) in zip(rows, lens, seqs):
        refs.append(R.attention(qf[at:at + n], k, v, length - n, mode == FA, SINK, WINDOW))
        at += n
    return lens, kv, pt, q, qf, seqs, np.concatenate([r[0] for r in refs]), np.concatenate([r[1] for r in refs])


DECODE = [
    # keys, hq, hkv, d
    ([7, 64, 65, 200, 31], 8, 2, 128),
    ([2001], 8, 2, 64),
    ([900, 5000, 3000], 28, 4, 128),
    ([700] * 40, 16, 8, 64),
    ([3000, 60], 40, 2, 128),                                # two blocks of queries
]


@pytest.mark.parametrize("mode", [FA, SA])
@pytest.mark.parametrize("case", DECODE, ids=[str(i) for i in range(len(DECODE))])
def test_decode_weights(F, ctx, case, mode):
    """fp32 outputs: three terms.  bf16 outputs are those, rounded once, but where two terms bring a result over the border: a step of it
    at most."""
    keys, hq, hkv, d = case
    rows = [1] * len(keys)
    lens, kv, pt, q, qf, seqs, ref, _ = case_of(F, rows, [n - 1 for n in keys], hq, hkv, d, mode, sum(keys))
    outs = []
    for fp32 in (1, 0):
        out = torch.empty(len(keys), hq, d, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
        F.flux_attn_decode_paged(ctx, F.attn_cfg(hq, hkv, d, SINK, WINDOW, 0.0, fp32), q, max(lens), kv, pt,
                                 torch.full((len(keys),), mode, dtype=torch.uint8, device="cuda"), out)
        outs.append(H.torch_to_f64(out))
    assert R.rel(outs[0], ref) <= R.THREE_TERMS
    v = max(float(np.abs(s[1]).max()) for s in seqs)
    assert (np.abs(outs[1] - ref) <= tolerance(qf, seqs, d) * v + 2.0 ** -8 * np.abs(ref)).all()
    assert R.rel(outs[1], outs[0]) <= R.ONE_TERM             # a rounding to bf16
    assert (outs[1] != R.to_bf16(outs[0])).mean() <= 0.02    # (5e-6 of steps of 2^-8: some per cent of a per cent; near zero more)


PREFILL = [
    # new rows, cached before them, hq, hkv, d
    ([70, 200, 33], [300, 0, 64], 8, 2, 128),
    ([130], [10], 7, 1, 64),
    ([20, 40], [7000, 900], 8, 2, 128),                      # pages shared out
]


@pytest.mark.parametrize("mode", [FA, SA])
@pytest.mark.parametrize("case", PREFILL, ids=[str(i) for i in range(len(PREFILL))])
def test_prefill_weights(F, ctx, case, mode):
    rows, past, hq, hkv, d = case
    lens, kv, pt, q, qf, seqs, ref, spread = case_of(F, rows, past, hq, hkv, d, mode, sum(past))
    v = max(float(np.abs(s[1]).max()) for s in seqs)
    for fp32 in (1, 0):
        out = torch.empty(sum(rows), hq, d, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
        F.flux_attn_prefill_paged(ctx, F.attn_cfg(hq, hkv, d, SINK, WINDOW, 0.0, fp32), q, cu_of(rows), max(rows), max(lens), kv, pt,
                                  torch.full((len(rows),), mode, dtype=torch.uint8, device="cuda"), out)
        got = H.torch_to_f64(out)
        bound = tolerance(qf, seqs, d) * v + 2.0 ** -8 / (1 - 2.0 ** -8) * spread
        bound = bound + (0 if fp32 else 2.0 ** -8 * (np.abs(ref) + bound))
        assert (np.abs(got - ref) <= bound).all()
        assert R.rel(got, ref) <= (R.ONE_TERM if fp32 else R.ONE_TERM_BF16)


@pytest.mark.parametrize("d", [64, 128])
def test_values_are_not_rounded(F, ctx, d):
    """Queries of zero see the mean of the values.  Lists of one page whose scale is no power of two: what the weights are rounded to is a
    factor of numerator and denominator alike, so fp32 sums are all that is left (64 terms each, and a handful of factors).  Values
    rounded to bf16 would be off by 2^-8 each."""
    hq, hkv, rows, lens = 8, 2, [2, 30, 1], [64, 37, 1]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=d, rows=rows)
    q.zero_()
    out = torch.empty(sum(rows), hq, d, dtype=torch.float32, device="cuda")
    F.flux_attn_prefill_paged(ctx, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1), q, cu_of(rows), 30, 64, kv, pt, torch.ones(3, dtype=torch.uint8, device="cuda"), out)
    got, at = H.torch_to_f64(out), 0
    for n, length, (_, v) in zip(rows, lens, seqs):
        for r in range(n):
            seen = np.repeat(v[:length - n + r + 1], hq // hkv, axis=1)
            assert (np.abs(got[at + r] - seen.mean(0)) <= (2 * 64 + 8) * 2.0 ** -24 * np.abs(seen).mean(0)).all()
        at += n


def test_parts_of_any_size_give_the_same_rows(F):
    """Workspaces without room for shared tiles, for some parts and for all that are worth it: whether the tiles are shared out depends on
    the room, so the sums differ, by no more than the roundings of the weights."""
    rows, past, hq, hkv, d = [20, 3], [7000, 5000], 8, 2, 128
    lens, kv, pt, q, qf, seqs, ref, spread = case_of(F, rows, past, hq, hkv, d, FA, 3)
    v = max(float(np.abs(s[1]).max()) for s in seqs)
    outs = []
    for room in (1, (8 << 20) + 8192 + 40 * 128 * 130 * 4, 0):
        c = F.flux_create(0, room)
        out = torch.empty(sum(rows), hq, d, dtype=torch.float32, device="cuda")
        F.flux_attn_prefill_paged(c, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1), q, cu_of(rows), 20, max(lens), kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
        outs.append(H.torch_to_f64(out))
        F.flux_destroy(c)
    for x in outs:
        assert (np.abs(x - ref) <= tolerance(qf, seqs, d) * v + 2.0 ** -8 / (1 - 2.0 ** -8) * spread).all()
        assert R.rel(x, ref) <= R.ONE_TERM
    assert not np.array_equal(outs[0], outs[2])
