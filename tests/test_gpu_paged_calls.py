"""Calls of the paged cache that its header allows and that the tests of its parts do not make: pools wider than 32-bit offsets, the smallest
bound of sparse layers, padded batches, a release that keeps everything."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from tests.test_gpu_paged import FA, SA, F, attention_case, bf16, check as check_decode, ctx, cu_of, decode_ref, i32, page_state, same_pages, tolerance  # noqa: F401
from tests.test_gpu_paged_prefill import check, prefill_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_a_pool_of_more_than_four_gigabytes(F, ctx, d):
    """Pages 1 GiB apart: what is written to the last ones and read from them lies behind 2^32 bytes."""
    hq, hkv, n_pages, wide, far = 8, 2, 6, 8, 1 << 30
    rng = np.random.default_rng(d)
    room = [torch.empty((n_pages - 1) * far + hkv * 64 * d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = (x.as_strided((n_pages, hkv, 64, d), (far, 64 * d, d, 1)) for x in room)
    scale = [torch.full((n_pages, hkv), float("nan"), device="cuda") for _ in range(2)]
    for x in (k, v):
        x.fill_(0x7F)
    kv, pt = F.PagedKV(k, v, *scale), F.PageTable.empty(2, n_pages, wide)
    o = P.Pages(pt.table.tolist(), [0, 0], pt.free_pages.tolist(), n_pages, n_pages)
    codes, scales = [np.full((n_pages, hkv, 64, d), 0x7F, np.uint8) for _ in range(2)], [np.full((n_pages, hkv), np.nan, np.float32) for _ in range(2)]
    cfg, mode = F.attn_cfg(hq, hkv, d, 4, 100, 0.0, 1), torch.tensor([FA, SA], dtype=torch.uint8, device="cuda")
    for rows in ([100, 200], [1, 1], [20, 30]):              # the second and the third go on in pages far behind
        t = sum(rows)
        slots = torch.empty(t, dtype=torch.int32, device="cuda")
        F.flux_page_plan(ctx, pt, cu_of(rows), t, slots)
        want, over = o.plan(rows)
        assert not over and slots.tolist() == want
        kn, kf = bf16(rng.standard_normal((t, hkv, d)) * 2.0 ** rng.integers(-2, 3, (t, 1, 1)))
        vn, vf = bf16(rng.standard_normal((t, hkv, d)))
        q, qf = bf16(rng.standard_normal((t, hq, d)))
        F.flux_kv_append_paged(ctx, kv, hkv, d, kn, vn, slots, t)
        for c, s, x in zip(codes, scales, (kf, vf)):
            P.append(c, s, x, want)
        seqs = [[P.gather(c, s, o.table[b], o.kv_len[b]) for c, s in zip(codes, scales)] for b in range(2)]
        out = torch.empty(t, hq, d, dtype=torch.float32, device="cuda")
        ref = prefill_ref(qf, seqs, rows, [FA, SA], 4, 100)
        F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), max(rows), 64 * wide, kv, pt, mode, out)   # (a run in the second step)
        check(out, ref, tolerance(qf, seqs, d), seqs)
        last = [rows[0] - 1, t - 1]
        one = torch.empty(2, hq, d, dtype=torch.float32, device="cuda")
        F.flux_attn_decode_paged(ctx, cfg, q[last].contiguous(), 64 * wide, kv, pt, mode, one)
        check_decode(one, ref[last], tolerance(qf, seqs, d), seqs)
    assert max(o.table[1]) == 5 and np.array_equal(k[5].cpu().numpy(), codes[0][5]) and np.array_equal(v[5].cpu().numpy(), codes[1][5])
    assert F.flux_last_device_status(ctx) == 0


@pytest.mark.parametrize("n_sink,window,block", [(0, 1, 0), (10, 70, 0), (64, 128, 0), (65, 129, 0), (10, 70, 16), (100, 200, 128), (1, 63, 0)])
def test_the_smallest_bound_of_sparse_layers(F, ctx, n_sink, window, block):
    """64 (ceil(n_sink / 64) + ceil(window / 64) + 1) is enough for decode, wherever the window lies in its pages."""
    up = lambda x: -(-x // max(1, block)) * max(1, block)
    bound = 64 * (-(-up(n_sink) // 64) + -(-up(window) // 64) + 1)
    lens = [2000 + i for i in range(0, 131, 5)] + [1, 64, 500]
    hq, hkv, d = 8, 2, 64
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=window)
    out = torch.empty(len(lens), hq, d, dtype=torch.float32, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, n_sink, window, 0.0, 1, block)
    F.flux_attn_decode_paged(ctx, cfg, q, bound, kv, pt, torch.zeros(len(lens), dtype=torch.uint8, device="cuda"), out)
    check_decode(out, decode_ref(qf, seqs, [SA] * len(lens), n_sink, window, max(1, block)), tolerance(qf, seqs, d), seqs)
    assert F.flux_last_device_status(ctx) == 0


def test_padded_batches(F, ctx):
    """Rows in front of the first sequence's and behind the last one's have no place, and sequences without rows and keys none in the result."""
    hq, hkv, d, rows = 8, 2, 64, [0, 40, 0, 3, 0]
    pt, o = page_state(F, [0, 50, 0, 64, 0], 4, 12, 5)
    t = 64
    cu = i32([5] + [5 + x for x in np.cumsum(rows)])
    slots = torch.full((t,), -9, dtype=torch.int32, device="cuda")
    F.flux_page_plan(ctx, pt, cu, t, slots)
    want, _ = o.plan(rows)
    want = [-1] * 5 + want + [-1] * (t - 5 - len(want))
    assert slots.tolist() == want
    same_pages(pt, o)
    codes, scale = [np.zeros((12, hkv, 64, d), np.uint8) for _ in range(2)], [np.ones((12, hkv), np.float32) for _ in range(2)]
    kv = F.PagedKV(*(torch.from_numpy(c).cuda() for c in codes), *(torch.from_numpy(s).cuda() for s in scale))
    rng = np.random.default_rng(1)
    kn, kf = bf16(rng.standard_normal((t, hkv, d)))
    kn[:5], kn[48:] = float("nan"), float("inf")             # padding may hold anything
    F.flux_kv_append_paged(ctx, kv, hkv, d, kn, kn, slots, t)
    for c, s, x in zip(codes, scale, (kv.k, kv.v)):
        P.append(c, s, kf, want)
        assert np.array_equal(x.cpu().numpy(), c)
    assert np.array_equal(kv.k_scale.cpu().numpy(), scale[0])
    q, qf = bf16(rng.standard_normal((t, hq, d)))
    cfg, mode = F.attn_cfg(hq, hkv, d, 4, 100, 0.0, 1), torch.tensor([1, 1, 0, 0, 1], dtype=torch.uint8, device="cuda")
    seqs = [[P.gather(c, s, o.table[b], o.kv_len[b]) for c, s in zip(codes, scale)] for b in range(5)]
    ref = np.zeros((t, hq, d))
    ref[5:48] = prefill_ref(qf[5:48], seqs, rows, mode.tolist(), 4, 100)
    out = torch.full((t, hq, d), 7.0, dtype=torch.float32, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu, 40, 256, kv, pt, mode, out)
    check(out[5:48], ref[5:48], tolerance(qf, seqs, d), seqs)
    assert (out[:5] == 7).all() and (out[48:] == 7).all()
    one = torch.full((7, hq, d), 7.0, dtype=torch.float32, device="cuda")
    F.flux_attn_decode_paged(ctx, cfg, q[:5], 256, kv, pt, mode, one[:5])
    check_decode(one[:5], decode_ref(qf[:5], seqs, mode.tolist(), 4, 100), tolerance(qf, seqs, d), seqs)
    assert (one[[0, 2, 4]] == 0).all() and (one[5:] == 7).all()
    # a release that keeps what there is, by the lengths themselves, and one by numbers beyond them
    before = [x.clone() for x in (pt.table, pt.kv_len, pt.free_pages, pt.n_free)]
    F.flux_page_release(ctx, pt, pt.kv_len)
    F.flux_page_release(ctx, pt, i32([2 ** 31 - 1] * 5))
    assert all(torch.equal(a, b) for a, b in zip(before, (pt.table, pt.kv_len, pt.free_pages, pt.n_free)))
    assert F.flux_last_device_status(ctx) == 0
