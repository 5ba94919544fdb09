"""Calls of the serving operators that programs make beside the ordinary ones: compaction in a captured graph, a fork and a compaction on another
stream, cross attention over scores that lie far apart, and over more rows than fit beside each other."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from tests.test_gpu_page_moves import fork_and_compare, state
from tests.test_gpu_paged import F, bf16, ctx, cu_of, i32, same_pages  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [300, 20000])
def test_forks_and_compactions_in_a_graph(F, ctx, n_pages):
    """Each replay forks, closes the holes and moves the codes; eager calls between."""
    b, hkv, d, wide = 6, 2, 64, 12
    pt, shares, o, os = state(F, [(3, [700, 650, 200]), (0, [64 * 11, 10, 300])], wide, n_pages, 3)
    codes = torch.randint(0, 0x7F, (2, n_pages, hkv, 64, d), dtype=torch.uint8, device="cuda")
    scales = torch.exp2(torch.randint(-9, -6, (2, n_pages, hkv), device="cuda").float())
    kv = F.PagedKV(codes[0], codes[1], scales[0], scales[1])
    ref = [(c.cpu().numpy().copy(), s.cpu().numpy().copy()) for c, s in zip(codes, scales)]
    parent, keep, copies, n = i32([0] * b), i32([0] * b), torch.empty(b, 3, dtype=torch.int32, device="cuda"), i32([0])
    moves, m = torch.empty(200, 3, dtype=torch.int32, device="cuda"), i32([0])

    def calls():
        F.flux_page_fork(ctx, pt, shares, parent, keep, copies, n)
        F.flux_page_copy(ctx, kv, hkv, d, copies, n)
        F.flux_page_compact(ctx, pt, shares, moves, m)
        F.flux_page_copy(ctx, kv, hkv, d, moves, m)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    rng = np.random.default_rng(8)
    for turn in range(6):
        p = list(range(b)) if turn == 0 else [int(x) for x in rng.integers(0, b, b)]
        size = [int(x) for x in rng.integers(1, 700, b)]
        parent.copy_(i32(p)), keep.copy_(i32(size))
        if turn % 2 == 0:
            graph.replay()
        else:
            calls()
        torch.cuda.synchronize()
        entries, short = S.fork(o, os, p, size)
        assert not short
        for c, s in ref:
            S.copy_pages(c, s, entries)
        moved = S.compact(o, os, 200)
        for c, s in ref:
            S.copy_pages(c, s, moved)
        same_pages(pt, o)
        assert shares.tolist() == os and int(n) == len(entries) and int(m) == len(moved)
        for got, got_scale, (c, s) in zip(codes, scales, ref):
            assert np.array_equal(got_scale.cpu().numpy(), s) and np.array_equal(got.cpu().numpy(), c)
    assert F.flux_last_device_status(ctx) == 0


def test_a_fork_on_another_stream(F, ctx):
    pt, shares, o, os = state(F, [(2, [200, 150, 130]), (0, [64, 70])], 6, 400, 5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fork_and_compare(F, ctx, pt, shares, o, os, [1, 1, 0, 4, -1], [199, 0, 130, 70, 3])
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["rising", "falling", "low", "one"])
@pytest.mark.parametrize("n,hq,hkv,d", [(1, 8, 2, 64), (6, 8, 2, 64), (6, 8, 8, 128), (130, 4, 4, 64), (200, 8, 2, 128)])
def test_cross_over_scores_far_apart(F, ctx, kind, n, hq, hkv, d):
    """Scores from some hundreds below zero to some hundreds above it, in either order; all of them hundreds below; one key that has all the weight."""
    rng, t = np.random.default_rng(n + d), 900
    q, qx = bf16(4.0 + rng.normal(size=(n, hq, d)) * 0.25)
    ramp = {"rising": np.linspace(-8, 8, t), "falling": np.linspace(8, -8, t), "low": np.full(t, -9.0), "one": np.where(np.arange(t) == 517, 8.0, -8.0)}[kind]
    k, kx = bf16(ramp[:, None] + rng.normal(size=(1, hkv, t, d)) * 0.25)
    v, vx = bf16(rng.normal(size=(1, hkv, t, d)))
    out = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
    F.flux_attn_cross(ctx, F.attn_cfg(hq, hkv, d, 0, 1), q, cu_of([n]), n, t, F.KVCache(k, v, i32([t])), out)
    ref, mag = S.cross(qx, kx[0].transpose(1, 0, 2), vx[0].transpose(1, 0, 2), 1 / np.sqrt(d))
    # as in tests/test_gpu_cross.py, with what fp32 leaves of scores of this size: each is a sum of d products, off by d * 2^-24 of their magnitudes,
    # and enters a weight and the sum of weights
    size = float(np.abs(qx).max() * np.abs(kx).max()) * d / np.sqrt(d)
    tol = (2 * 2.0 ** -8 + 2 * d * 2.0 ** -24 * size) * mag + 2.0 ** -8 * np.abs(ref) + 1e-30
    off = np.abs(out.double().cpu().numpy() - ref)
    assert (off <= tol).all(), float((off / tol).max())
    assert F.flux_last_device_status(ctx) == 0
