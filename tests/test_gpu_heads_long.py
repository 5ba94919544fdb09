"""Long calls of the appends with norm and rotation, blocks that are shared out differently over a launch, other streams, and captured calls."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from oracle import serving_oracle as S
from tests.test_gpu_heads import EPS, append_case, bf16, freqs, i32, near_enough, pool_of, rows, weights
from tests.test_gpu_paged import F, ctx, cu_of  # noqa: F401

pytestmark = pytest.mark.gpu


def paged_case(F, ctx, t, new, first, hq, hkv, d, rot, near, norm, seed=0, check_rows=None, stream=None):
    """One call, all pages and scales against the oracle; check_rows: of these queries only (all by default)."""
    _, _, (q, k, v), (qx, kx, vx) = rows(seed + t, t, hq, hkv, d)
    (wq, wk), (wqx, wkx) = weights(seed + t, d, norm)
    f, fx = freqs(rot) if rot else (None, None)
    held = [-(-(a + b) // 64) for a, b in zip(first, new)]
    ids = np.random.default_rng(seed + t).permutation(sum(held) + 2)
    slots, at = [], 0
    for n, r, h in zip(new, first, held):
        slots.append(ids[at + (r + np.arange(n)) // 64] * 64 + (r + np.arange(n)) % 64)
        at += h
    slots = np.concatenate(slots)
    pos = np.random.default_rng(seed + t).integers(0, 100000, t)
    kv, codes, scales = pool_of(F, seed + t, sum(held) + 2, hkv, d)
    out = torch.full((t + 1, hq, d), -7.0, dtype=torch.bfloat16, device="cuda")
    args = (F.head_cfg(hq, hkv, d, wq, wk, EPS, f, rot, near), kv, q, k, v, i32(slots), i32(pos) if rot else None, t, out)
    if stream is None:
        F.flux_qkv_append_paged(ctx, *args)
    else:
        stream.wait_stream(torch.cuda.current_stream())
        F.flux_qkv_append_paged(ctx, *args, stream=stream)
        stream.synchronize()
    at = np.arange(t) if check_rows is None else check_rows
    n = S.normed(qx[at], wqx, EPS)
    near_enough(out[torch.from_numpy(at).cuda()], n if not rot else S.turned(n, pos[at], fx, near), n, rot, near)
    assert bool((out[t] == -7.0).all())
    want = S.heads(kx, wkx, EPS, pos, fx, near)
    for got, got_scale, c, s, y in ((kv.k, kv.k_scale, codes[0], scales[0], want), (kv.v, kv.v_scale, codes[1], scales[1], vx)):
        P.append(c, s, y, slots)
        assert np.array_equal(got_scale.cpu().numpy(), s)
        assert np.array_equal(got.cpu().numpy() & 0x7F, c & 0x7F) and np.array_equal(P.VALUES[got.cpu().numpy()], P.VALUES[c])
    assert F.flux_last_device_status(ctx) == 0


@pytest.mark.parametrize("new,first,hq,hkv,d,rot,near,norm", [
    ([1000, 1100], [5, 60], 2, 2, 64, 64, 0, True),                      # long blocks, K and V apart
    ([1] * 1500, [i % 64 for i in range(1500)], 1, 3, 64, 32, 1, True),  # a block a row, 64 of them in a tile
    ([3] * 200 + [64, 1, 200, 31, 33, 32], [63] * 200 + [0, 5, 1, 32, 31, 33], 4, 2, 128, 128, 0, True),
    ([8, 9] * 40, [0] * 80, 3, 17, 64, 64, 0, False),                    # blocks about as long as one wave takes alone, an odd number of heads
    ([16, 17, 7] * 12, [50] * 36, 3, 17, 128, 48, 1, True),
    ([70], [3], 1, 40, 64, 0, 0, True),
    ([1] * 130, [(i * 5) % 64 for i in range(130)], 2, 17, 64, 64, 0, True),      # single rows, heads that do not fill the last wave
    ([1, 2, 1, 9, 1, 1] * 9, [(i * 7) % 64 for i in range(54)], 1, 11, 128, 64, 1, True),
    ([1] * 40, [63, 0] * 20, 3, 24, 128, 0, 0, False),
    ([8192 + 31], [17], 1, 1, 64, 64, 0, True),                          # as many tiles as workgroups side by side, and more
    ([8100, 8300], [0, 40], 1, 2, 128, 128, 0, True),
    ([1] * 64 + [16500], list(range(64)) + [9], 1, 3, 64, 64, 0, False),
])
def test_append_paged_long(F, ctx, new, first, hq, hkv, d, rot, near, norm):
    t = sum(new)
    paged_case(F, ctx, t, new, first, hq, hkv, d, rot, near, norm, check_rows=np.unique(np.linspace(0, t - 1, 500).astype(int)))


def test_append_paged_on_another_stream(F, ctx):
    paged_case(F, ctx, 200, [150, 50], [0, 9], 4, 2, 64, 64, 0, True, stream=torch.cuda.Stream())


def test_heads_of_many_rows(F, ctx):
    """More rows than a launch has waves, a token's heads that do not fill its last wave."""
    t, hq, hkv, d = 9001, 5, 2, 64
    _, _, (q, k, _), (qx, kx, _) = rows(1, t, hq, hkv, d)
    (wq, wk), (wqx, wkx) = weights(1, d)
    f, fx = freqs(48)
    pos = np.arange(t)
    qo, ko = (torch.full((t + 1, h, d), -7.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
    F.flux_qk_norm_rope(ctx, F.head_cfg(hq, hkv, d, wq, wk, EPS, f, 48, 1), q, k, i32(pos), t, qo, ko)
    for got, y, w in ((qo, qx, wqx), (ko, kx, wkx)):
        n = S.normed(y, w, EPS)
        near_enough(got[:t], S.turned(n, pos, fx, True), n, 48, True)
        assert bool((got[t:] == -7.0).all())


def test_append_of_many_sequences(F, ctx):
    """More sequences than a lane search takes in one step, most of them without a row; lengths that are loaded ahead and lengths that are not."""
    rng = np.random.default_rng(7)
    for n in (65, 256, 257, 700):
        new = rng.integers(0, 3, n)
        append_case(F, ctx, n, rng.integers(0, 6, n).tolist(), new.tolist(), 3, 1, 64, 64, 0, True, 9)


def test_append_of_long_chunks(F, ctx):
    append_case(F, ctx, 3, [0, 17, 2, 0], [3000, 1, 2049, 0], 4, 2, 128, 128, 0, True, 3100)


def test_captured_appends(F, ctx):
    """A step of both caches as a graph, replayed with eager calls between: every replay appends behind the rows of the one before."""
    b, hq, hkv, d, cap, steps = 5, 4, 2, 64, 80, 4
    dev, x, (q, k, v), (qx, kx, vx) = rows(1, b, hq, hkv, d)
    (wq, wk), (wqx, wkx) = weights(1, d)
    f, fx = freqs(64)
    hc = F.head_cfg(hq, hkv, d, wq, wk, EPS, f)
    held = torch.zeros(2, b, hkv, cap, d, dtype=torch.bfloat16, device="cuda")
    lens = i32([3, 0, 62, 10, 63])
    cache = F.KVCache(held[0], held[1], lens)
    kv, codes, scales = pool_of(F, 1, 2 * b, hkv, d)
    slots, pos, cu = i32([0] * b), i32([0] * b), cu_of([1] * b)
    out, out2 = (torch.zeros(b, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step():
        F.flux_qkv_append(ctx, hc, cache, q, k, v, cu, b, 1, None, out)
        F.flux_qkv_append_paged(ctx, hc, kv, q, k, v, slots, pos, b, out2)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    at = np.array([3, 0, 62, 10, 63])
    for i in range(2 * steps):
        new, _ = bf16(np.random.default_rng(50 + i).normal(size=(b, hq + 2 * hkv, d)))
        dev.copy_(new)
        x = dev.double().cpu().numpy()
        row = (2 * np.arange(b) + at // 64) * 64 + at % 64
        slots.copy_(i32(row))
        pos.copy_(i32(at))
        if i % 2:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        n = S.normed(x[:, :hq], wqx, EPS)
        for o in (out, out2):
            near_enough(o, S.turned(n, at, fx, False), n, 64, False)
        key = S.normed(x[:, hq:hq + hkv], wkx, EPS)
        near_enough(held[0][torch.arange(b), :, torch.from_numpy(at).cuda()], S.turned(key, at, fx, False), key, 64, False)
        assert torch.equal(held[1][torch.arange(b), :, torch.from_numpy(at).cuda()], dev[:, hq + hkv:])
        want = S.heads(x[:, hq:hq + hkv], wkx, EPS, at, fx, False)
        for got, got_scale, c, s, y in ((kv.k, kv.k_scale, codes[0], scales[0], want), (kv.v, kv.v_scale, codes[1], scales[1], x[:, hq + hkv:])):
            P.append(c, s, y, row.tolist())
            assert np.array_equal(got_scale.cpu().numpy(), s)
            assert np.array_equal(P.VALUES[got.cpu().numpy()], P.VALUES[c])
        at = at + 1
        assert lens.tolist() == at.tolist()
    assert F.flux_last_device_status(ctx) == 0


def test_single_rows_without_norm_as_the_plain_call(F, ctx):
    """One row of many sequences, values that are not finite among them, pages that take a larger scale: the pages of flux_kv_append_paged, bit for bit."""
    t, hkv = 70, 11
    for d in (64, 128):
        _, x, _, _ = rows(d, t, 1, hkv, d)
        x[3, 1, 7], x[40, 2, 9], x[66, 13, 0], x[69, 22, 1], x[5, 12, :] = np.inf, np.nan, -np.inf, 1e30, 300.0
        dev, _ = bf16(x)
        k, v = dev[:, 1:1 + hkv], dev[:, 1 + hkv:]
        slots = i32([64 * i + (i * 11) % 64 for i in range(t)])
        a, _, _ = pool_of(F, 1, t, hkv, d)
        b, _, _ = pool_of(F, 1, t, hkv, d)
        F.flux_qkv_append_paged(ctx, F.head_cfg(1, hkv, d), a, None, k, v, slots, None, t, None)
        F.flux_kv_append_paged(ctx, b, hkv, d, k.contiguous(), v.contiguous(), slots, t)
        for p, q in ((a.k, b.k), (a.v, b.v)):
            assert bool(((p == q) | (((p & 0x7F) == 0x7F) & ((q & 0x7F) == 0x7F))).all())     # (the sign of NaN is nobody's)
        assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)
