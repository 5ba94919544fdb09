"""Prefill attention over the paged 8-bit cache against the float64 oracle, and the calls of the paged cache together as a
serving program makes them."""
import numpy as np
import pytest
import torch

from oracle import flux_oracle as O
from oracle import paged_oracle as P
from tests import helpers as H
from tests.test_gpu_paged import FA, SA, F, attention_case, bf16, ctx, cu_of, i32, paged_kv, tolerance  # noqa: F401

pytestmark = pytest.mark.gpu


def prefill_ref(qf, seqs, rows, modes, n_sink, window, block=1, scale=None):
    out, at = np.zeros(qf.shape), 0
    for b, (k, v) in enumerate(seqs):
        n = min(rows[b], len(k))
        if n:
            out[at:at + n] = O.attention(qf[at:at + n], k, v, modes[b], n_sink, window, scale, block=block)
        at += rows[b]
    return out


def check(out, ref, eps, seqs):
    """As for decode, but weights are rounded to bf16 (2^-8 of each, in numerator and denominator alike: 2 * 2^-8 of the largest |v|
    at most) and so are values whose scale is no power of two (2^-8 of |v|).  Of the 2-norm the roundings of weights, values and bf16
    outputs take 2^-8 each at most, and are independent: below 2^-7 together."""
    got = H.torch_to_f64(out)
    assert np.isfinite(got).all()
    v = max(float(np.abs(s[1]).max()) if s[1].size else 0.0 for s in seqs)
    bound = (eps + 3 * 2.0 ** -8) * v + (2.0 ** -8 * np.abs(ref) if out.dtype == torch.bfloat16 else 0)
    assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) - bound).max())
    rel = np.sqrt(((got - ref) ** 2).sum() / max((ref ** 2).sum(), 1e-300))
    assert rel <= 2.0 ** -7, rel


CASES = [
    # new rows, cached before them, modes, hq, hkv, d, n_sink, window, sa_block
    ([1], [0], [FA], 1, 1, 64, 0, 1, 0),
    ([1, 0, 5, 64], [0, 3, 60, 64], [FA] * 4, 4, 2, 128, 4, 16, 0),
    ([63, 64, 65, 130], [0, 0, 0, 0], [FA, FA, SA, SA], 8, 2, 64, 4, 16, 0),
    ([200, 333], [0, 100], [SA, FA], 14, 2, 128, 10, 100, 0),                # group 7
    ([257, 100, 300], [0, 700, 129], [SA, SA, SA], 8, 2, 128, 16, 128, 64),
    ([40, 500], [1000, 0], [SA, SA], 4, 4, 64, 130, 70, 16),                  # group 1; sinks of two pages and two positions
    ([5] * 6, [300, 2000, 64, 63, 4000, 1], [FA, SA, FA, FA, FA, SA], 32, 8, 128, 128, 512, 0),   # drafts: pages are shared out
    ([3], [6000], [FA], 16, 1, 128, 0, 1, 0),                                 # one KV head, group 16
    ([2], [6000], [SA], 16, 1, 128, 70, 300, 0),                              # ... two blocks of columns
    ([4, 0, 1, 3], [700, 500, 20000, 64], [FA, FA, SA, SA], 8, 2, 64, 5, 100, 0),     # runs of uneven length, one block
    ([1, 8, 2, 7, 8], [64, 511, 448, 3000, 62], [SA, SA, FA, SA, FA], 8, 2, 128, 3, 64, 64),   # runs across page borders
    ([8, 8], [100000, 3], [FA, FA], 4, 1, 64, 0, 1, 0),
    ([1 + i % 5 for i in range(64)], [(i * 97) % 900 + 1 for i in range(64)], [i % 2 for i in range(64)], 12, 2, 128, 3, 70, 0),
    ([17, 1], [5000, 9000], [FA, SA], 40, 2, 64, 64, 3000, 0),                # group 20
    ([600], [1500], [FA], 8, 2, 128, 0, 1, 0),
    ([900], [0], [SA], 8, 1, 64, 2 ** 31 - 1, 2 ** 31 - 1, 64),               # the sparse rule sees everything
    ([1 + i % 9 for i in range(130)], [i * 7 % 300 for i in range(130)], [i % 2 for i in range(130)], 4, 2, 64, 3, 70, 0),
    ([300], [40], [SA], 6, 3, 128, 0, 1, 0),                                  # a window of one, no sinks
]


@pytest.mark.parametrize("fp32", [1, 0])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_prefill_against_the_oracle(F, ctx, case, fp32):
    rows, past, modes, hq, hkv, d, n_sink, window, block = case
    lens = [a + b for a, b in zip(rows, past)]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, ("phtd", "pthd", "wide")[len(lens) % 3], seed=sum(lens) + d, rows=rows)
    guard = torch.full((sum(rows) + 2, hq, d), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, n_sink, window, 0.0, fp32, block)
    mode = torch.tensor(modes, dtype=torch.uint8, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), max(rows), max(lens), kv, pt, mode, guard[1:-1])
    ref = prefill_ref(qf, seqs, rows, modes, n_sink, window, max(1, block))
    check(guard[1:-1], ref, tolerance(qf, seqs, d), seqs)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    assert F.flux_last_device_status(ctx) == 0
    again = torch.empty_like(guard[1:-1])
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), max(rows), max(lens), kv, pt, mode, again)
    assert torch.equal(again, guard[1:-1])
    # loose bounds are as good, and so is a workspace without room for shared tiles
    wide = 64 * pt.table.shape[1]
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), wide, wide, kv, pt, mode, again)
    check(again, ref, tolerance(qf, seqs, d), seqs)
    small = F.flux_create(0, 1)
    F.flux_attn_prefill_paged(small, cfg, q, cu_of(rows), max(rows), max(lens), kv, pt, mode, again)
    check(again, ref, tolerance(qf, seqs, d), seqs)
    torch.cuda.synchronize()
    F.flux_destroy(small)


def test_prefill_with_power_of_two_scales_and_a_workspace_for_few_parts(F):
    """The scales that the append writes are exact in bf16: values are not rounded then.  A workspace that holds some parts makes the
    parts longer."""
    rows, past, hq, hkv, d = [20, 3], [7000, 5000], 8, 2, 128
    lens = [a + b for a, b in zip(rows, past)]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=3, rows=rows)
    for t in (kv.k_scale, kv.v_scale):
        t.copy_(torch.exp2(torch.floor(torch.log2(t))))
    codes = [x.cpu().numpy() for x in (kv.k, kv.v)]
    scale = [x.cpu().numpy() for x in (kv.k_scale, kv.v_scale)]
    table = pt.table.cpu().numpy()
    seqs = [[P.gather(c, s, table[b], n) for c, s in zip(codes, scale)] for b, n in enumerate(lens)]
    ref = prefill_ref(qf, seqs, rows, [FA, FA], 0, 1)
    outs = []
    for room in (0, (8 << 20) + 4096 + 40 * 128 * 130 * 4, (8 << 20) + 4096 + 200 * 128 * 130 * 4):
        c = F.flux_create(0, room)
        out = torch.empty(sum(rows), hq, d, dtype=torch.float32, device="cuda")
        F.flux_attn_prefill_paged(c, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1), q, cu_of(rows), 20, max(lens), kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
        check(out, ref, tolerance(qf, seqs, d), seqs)
        outs.append(out)
        torch.cuda.synchronize()
        F.flux_destroy(c)


def test_prefill_where_pages_are_missing_and_lengths_do_not_fit(F, ctx):
    hq, hkv, d = 8, 2, 128
    rows, lens = [10, 100, 6], [300, 200, 64]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=9, rows=rows)
    pt.table[0, 1], pt.table[0, 4], pt.table[2, 0] = -1, kv.k.shape[0], 2 ** 31 - 1
    out = torch.full((116, hq, d), 7.0, dtype=torch.float32, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1)
    mode = torch.ones(3, dtype=torch.uint8, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), 100, 300, kv, pt, mode, out)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    ref = prefill_ref(qf, seqs, rows, [FA] * 3, 0, 1)
    k, v = (x[np.r_[0:64, 128:256]] for x in seqs[0])        # sequence 0 sees these, all of them before its queries
    for h in range(hq):
        s = qf[:10, h] @ k[:, h // 4].T / np.sqrt(d)
        p = np.exp(s - s.max(1, keepdims=True))
        ref[:10, h] = p @ v[:, h // 4] / p.sum(1, keepdims=True)
    ref[110:] = 0
    check(out, ref, tolerance(qf, seqs, d), seqs)
    assert (out[110:] == 0).all()
    # more queries than cached positions: the first kv_len rows, the others as they were
    kv, pt, q, qf, seqs = attention_case(F, [5, 40], hq, hkv, d, seed=2, rows=[9, 40])
    out = torch.full((49, hq, d), 7.0, dtype=torch.float32, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of([9, 40]), 40, 40, kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    check(out[:5], prefill_ref(qf[:5], seqs[:1], [5], [FA], 0, 1), tolerance(qf, seqs, d), seqs)
    check(out[9:], prefill_ref(qf[9:], seqs[1:], [40], [FA], 0, 1), tolerance(qf, seqs, d), seqs)
    assert (out[5:9] == 7).all()
    pt.kv_len[0], pt.kv_len[1] = -4, 10 ** 9                 # clamped to nothing, and to what the table holds
    pt.table.clamp_(0, kv.k.shape[0] - 1)
    kv.k.fill_(0)
    kv.v.fill_(0)
    kv.k_scale.fill_(1)
    kv.v_scale.fill_(1)
    F.flux_attn_prefill_paged(ctx, cfg, q, i32([0, -3, 9]), 40, 40, kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
    assert F.flux_last_device_status(ctx) & F.FLUX_DEV_BAD_LENGTH


@pytest.mark.parametrize("n", [2, 60])
def test_prefill_says_when_a_bound_is_too_low(F, ctx, n):
    hq, hkv, d = 8, 2, 64
    kv, pt, q, qf, seqs = attention_case(F, [1000, 640], hq, hkv, d, seed=9, rows=[n, n])
    out = torch.full((2 * n, hq, d), 7.0, dtype=torch.float32, device="cuda")
    F.flux_attn_prefill_paged(ctx, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1), q, cu_of([n, n]), n, 640, kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    check(out[n:], prefill_ref(qf[n:], seqs[1:], [n], [FA], 0, 1), tolerance(qf, seqs, d), seqs)
    assert torch.isfinite(out).all()
    out.fill_(7.0)                                           # rows beyond max_q_len are not computed, whatever tile they share
    F.flux_attn_prefill_paged(ctx, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1), q, cu_of([n, n]), 1, 1000, kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
    assert F.flux_last_device_status(ctx) == 0
    ref = prefill_ref(qf, seqs, [n, n], [FA, FA], 0, 1)
    check(out[[0, n]], ref[[0, n]], tolerance(qf, seqs, d), seqs)


@pytest.mark.parametrize("mode", [FA, SA])
def test_long_lists_of_many_tiles_are_shared_out(F, ctx, mode):
    """512 tiles of 128 to 160 pages, of which 768 run side by side, and the last tile of three tokens."""
    n, past, heads, d, sink, window = 4096 + 3, 6000, 16, 64, 70, 5000
    kv, pt, q, qf, seqs = attention_case(F, [past + n], heads, heads, d, seed=4, rows=[n])
    cfg, modes = F.attn_cfg(heads, heads, d, sink, window), torch.tensor([mode], dtype=torch.uint8, device="cuda")
    out = torch.full((n, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of([n]), n, past + n, kv, pt, modes, out)
    k, v = seqs[0]
    i, j = past + torch.arange(n, device="cuda")[:, None], torch.arange(past + n, device="cuda")[None]
    seen = (j <= i) & ((j < sink) | (i - j < window) | (mode == FA))
    bound = tolerance(qf, seqs, d)
    for h in (0, 9):                                         # the definition in float64, a head at a time
        kh, vh = (torch.from_numpy(np.ascontiguousarray(x[:, h])).cuda() for x in (k, v))
        s = (q[:, h].double() @ kh.T.contiguous() / d ** 0.5).masked_fill_(~seen, -torch.inf)
        ref = (torch.softmax(s, 1) @ vh).cpu().numpy()
        check(out[:, h], ref, bound, seqs)
    small = F.flux_create(0, 1)                              # without room for shared tiles: the same but for roundings
    again = torch.empty_like(out)
    F.flux_attn_prefill_paged(small, cfg, q, cu_of([n]), n, past + n, kv, pt, modes, again)
    v_max = float(np.abs(v).max())
    assert float((again.float() - out.float()).abs().max()) <= 2 * (bound + 3 * 2.0 ** -8 + 2.0 ** -8) * v_max
    assert F.flux_last_device_status(ctx) == 0
    torch.cuda.synchronize()
    F.flux_destroy(small)


def test_prefill_rows_are_those_of_decode(F, ctx):
    """The last query of a prefill call is the query of a decode call: the same to what the weights' rounding leaves."""
    hq, hkv, d = 16, 4, 128
    rows, lens = [70, 3], [1500, 900]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=12, rows=rows)
    cfg = F.attn_cfg(hq, hkv, d, 32, 200, 0.0, 1)
    mode = torch.tensor([0, 1], dtype=torch.uint8, device="cuda")
    out = torch.empty(73, hq, d, dtype=torch.float32, device="cuda")
    one = torch.empty(2, hq, d, dtype=torch.float32, device="cuda")
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), 70, 1500, kv, pt, mode, out)
    F.flux_attn_decode_paged(ctx, cfg, q[[69, 72]].contiguous(), 1500, kv, pt, mode, one)
    v = max(float(np.abs(s[1]).max()) for s in seqs)
    assert float((out[[69, 72]] - one).abs().max()) <= (2 * tolerance(qf, seqs, d) + 3 * 2.0 ** -8) * v


# ---- together --------------------------------------------------------------------------------------------------------

def test_serving_run(F, ctx):
    """Two layers, three requests: prompts in chunks, decode steps, drafted tokens of which some are rejected, a request that ends and
    another one that takes its row: every output against the oracle on what the pages stand for, every pool bit for bit."""
    rng = np.random.default_rng(77)
    layers, B, hq, hkv, d, n_sink, window, n_pages, wide = 2, 3, 8, 2, 64, 16, 100, 40, 16
    cfg = F.attn_cfg(hq, hkv, d, n_sink, window, 0.0, 1)
    pt = F.PageTable.empty(B, n_pages, wide)
    o = P.Pages(pt.table.tolist(), [0] * B, pt.free_pages.tolist(), n_pages, n_pages)
    modes = [[FA, SA, FA], [SA, SA, FA]]
    mode = torch.tensor(modes, dtype=torch.uint8, device="cuda")
    pools = [F.PagedKV.empty(n_pages, hkv, d) for _ in range(layers)]
    for kv in pools:                                         # (as allocated, memory may hold anything)
        for t in (kv.k, kv.v):
            t.view(torch.uint8).fill_(0x7F)
        kv.k_scale.fill_(float("nan"))
        kv.v_scale.fill_(float("nan"))
    codes = [[np.full((n_pages, hkv, 64, d), 0x7F, np.uint8) for _ in range(2)] for _ in range(layers)]
    scale = [[np.full((n_pages, hkv), np.nan, np.float32) for _ in range(2)] for _ in range(layers)]

    def step(rows, attend):
        t = sum(rows)
        slots = torch.empty(t, dtype=torch.int32, device="cuda")
        F.flux_page_plan(ctx, pt, cu_of(rows), t, slots)
        want, over = o.plan(rows)
        assert not over and slots.tolist() == want
        for i in range(layers):
            k, kf = bf16(rng.standard_normal((t, hkv, d)) * 2.0 ** rng.integers(-2, 3, (t, 1, 1)))
            v, vf = bf16(rng.standard_normal((t, hkv, d)))
            q, qf = bf16(rng.standard_normal((t, hq, d)))
            F.flux_kv_append_paged(ctx, pools[i], hkv, d, k, v, slots, t)
            for c, s, x in zip(codes[i], scale[i], (kf, vf)):
                P.append(c, s, x, want)
            out = torch.empty(t, hq, d, dtype=torch.float32, device="cuda")
            attend(i, q, out, rows)
            seqs = [[P.gather(c, s, o.table[b], o.kv_len[b]) for c, s in zip(codes[i], scale[i])] for b in range(B)]
            check(out, prefill_ref(qf, seqs, rows, modes[i], n_sink, window), tolerance(qf, seqs, d), seqs)
            for name, c in (("k", codes[i][0]), ("v", codes[i][1])):
                assert np.array_equal(getattr(pools[i], name).view(torch.uint8).cpu().numpy(), c), (i, name)
        assert pt.kv_len.tolist() == o.kv_len and pt.table.tolist() == o.table

    def prefill(i, q, out, rows):
        F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), max(rows), max(o.kv_len), pools[i], pt, mode[i], out)

    def decode(i, q, out, rows):
        F.flux_attn_decode_paged(ctx, cfg, q, max(o.kv_len), pools[i], pt, mode[i], out)

    def release(keep):
        F.flux_page_release(ctx, pt, i32(keep))
        o.release(keep)
        assert pt.table.tolist() == o.table and pt.free_pages.tolist() == o.free and pt.n_free.tolist() == [o.n_free]

    step([100, 3, 0], prefill)
    step([130, 61, 200], prefill)
    for _ in range(3):
        step([1, 1, 1], decode)
    step([5, 5, 5], prefill)                                 # drafts ...
    release([o.kv_len[0] - 4, o.kv_len[1], o.kv_len[2] - 2])   # ... some of them rejected
    step([1, 1, 1], decode)
    release([o.kv_len[0], 0, o.kv_len[2]])                   # request 1 ends, another one begins
    step([1, 310, 1], prefill)
    step([1, 1, 1], decode)
    assert F.flux_last_device_status(ctx) == 0


def test_a_step_replays_from_a_graph(F, ctx):
    """Plan, append and attention are launches on the caller's stream: captured once, replayed with the program's own work and
    eager calls between, every replay against the oracle."""
    rng = np.random.default_rng(5)
    B, hq, hkv, d, n_pages, wide = 2, 8, 2, 128, 30, 12
    cfg = F.attn_cfg(hq, hkv, d, 4, 100, 0.0, 1)
    pt = F.PageTable.empty(B, n_pages, wide)
    o = P.Pages(pt.table.tolist(), [0] * B, pt.free_pages.tolist(), n_pages, n_pages)
    kv = F.PagedKV.empty(n_pages, hkv, d)
    codes = [np.zeros((n_pages, hkv, 64, d), np.uint8) for _ in range(2)]
    scale = [np.ones((n_pages, hkv), np.float32) for _ in range(2)]
    mode = torch.tensor([1, 0], dtype=torch.uint8, device="cuda")
    rows = [1, 1]
    cu, keep = cu_of(rows), i32([10 ** 6] * B)
    slots = torch.empty(2, dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(2, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(2, hq, d, dtype=torch.bfloat16, device="cuda")
    out, out_p = (torch.zeros(2, hq, d, dtype=torch.float32, device="cuda") for _ in range(2))

    def calls():
        F.flux_page_release(ctx, pt, keep)
        F.flux_page_plan(ctx, pt, cu, 2, slots)
        F.flux_kv_append_paged(ctx, kv, hkv, d, k, v, slots, 2)
        F.flux_attn_decode_paged(ctx, cfg, q, 64 * wide, kv, pt, mode, out)
        F.flux_attn_prefill_paged(ctx, cfg, q, cu, 1, 64 * wide, kv, pt, mode, out_p)

    def fill():
        res = []
        for t in (k, v, q):
            x, xf = bf16(rng.standard_normal(t.shape))
            t.copy_(x)
            res.append(xf)
        return res

    def verify(kf, vf, qf):
        want, _ = o.plan(rows)
        P.append(codes[0], scale[0], kf, want)
        P.append(codes[1], scale[1], vf, want)
        seqs = [[P.gather(c, s, o.table[b], o.kv_len[b]) for c, s in zip(codes, scale)] for b in range(B)]
        ref = prefill_ref(qf, seqs, rows, [1, 0], 4, 100)
        for x in (out, out_p):
            check(x, ref, tolerance(qf, seqs, d), seqs)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                            # a first prompt, eagerly on another stream than the default one
        n = [500, 130]
        t = sum(n)
        s0 = torch.empty(t, dtype=torch.int32, device="cuda")
        x, xf = bf16(rng.standard_normal((t, hkv, d)))
        F.flux_page_plan(ctx, pt, cu_of(n), t, s0)
        F.flux_kv_append_paged(ctx, kv, hkv, d, x, x, s0, t)
    torch.cuda.current_stream().wait_stream(side)
    want, _ = o.plan(n)
    for c, s in zip(codes, scale):
        P.append(c, s, xf, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(5):
        f = fill()
        if turn == 2:
            calls()                                          # an eager step between replays
        else:
            graph.replay()
        torch.cuda.synchronize()
        verify(*f)
    assert F.flux_last_device_status(ctx) == 0


def test_lists_in_parts_from_a_graph_and_on_two_streams(F):
    """Calls whose lists are shared out and merged (tiles, runs of drafts, decode) give the same bits eagerly, replayed from a graph with other
    lengths than it was captured with, and with another context's calls on another stream beside them."""
    hq, hkv, d, rows = 8, 2, 128, [20, 3, 9]
    lens = [7000, 900, 3100]
    kv, pt, q, _, _ = attention_case(F, lens, hq, hkv, d, seed=21, rows=rows)
    cfg, wide = F.attn_cfg(hq, hkv, d, 16, 500), 64 * pt.table.shape[1]
    mode = torch.tensor([FA, SA, FA], dtype=torch.uint8, device="cuda")
    cu, cu_few = cu_of(rows), cu_of([4, 3, 4])

    def outputs():
        return [torch.zeros(sum(rows), hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(3)]

    def calls(ctx, out):
        F.flux_attn_prefill_paged(ctx, cfg, q, cu, 20, wide, kv, pt, mode, out[0])
        F.flux_attn_prefill_paged(ctx, cfg, q, cu_few, 4, wide, kv, pt, mode, out[1])
        F.flux_attn_decode_paged(ctx, cfg, q, wide, kv, pt, mode, out[2])

    states = [lens, [64, 900, 20], [6500, 7, 3000], [1, 0, 9]]   # (runs longer than their lists are cut)
    a, b = F.flux_create(0, 0), F.flux_create(0, 0)
    want = []
    for s in states:
        pt.kv_len.copy_(i32(s))
        out = outputs()
        calls(a, out)
        torch.cuda.synchronize()
        want.append(out)
    F.flux_last_device_status(a)
    out = outputs()
    graph = torch.cuda.CUDAGraph()
    pt.kv_len.copy_(i32(states[1]))
    with torch.cuda.graph(graph):
        calls(a, out)
    for turn in (0, 1, 2, 3, 0, 2):
        pt.kv_len.copy_(i32(states[turn]))
        for x in out:
            x.zero_()
        other = outputs()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(3):
                calls(b, other)
        graph.replay()
        torch.cuda.synchronize()
        for x, y, z in zip(out, want[turn], other):
            assert torch.equal(x, y) and torch.equal(z, y), turn
    for c in (a, b):
        F.flux_destroy(c)
