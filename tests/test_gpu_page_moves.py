"""Pages that change hands, move and are copied, on the GPU, against their plain definitions on lists; and a run of the calls of a
serving program together."""
import numpy as np
import pytest
import torch

from oracle import flux_oracle as O
from oracle import paged_oracle as P
from oracle import serving_oracle as S
from tests.test_gpu_heads import freqs, rows, weights
from tests.test_gpu_paged import F, ctx, cu_of, i32, same_pages  # noqa: F401

pytestmark = pytest.mark.gpu


def state(F, groups, table_pages, n_pages, seed):
    """Groups of (pages that all of them share, lengths): tables on shuffled pages, holders, and the same on lists."""
    ids = [int(x) for x in np.random.default_rng(seed).permutation(n_pages)]
    table, lens, shares, at = [], [], [0] * n_pages, 0
    for shared, sizes in groups:
        common, at = ids[at:at + shared], at + shared
        for p in common:
            shares[p] = len(sizes) - 1
        for n in sizes:
            own = S.pages_of(n) - shared
            assert own >= 0
            row, at = common + ids[at:at + own], at + own
            table.append(row + [-1] * (table_pages - len(row)))
            lens.append(n)
    free = ids[at:] + [-7] * at
    pt = F.PageTable(i32(table), i32(lens), i32(free), i32([n_pages - at]))
    return pt, i32(shares), P.Pages(table, lens, free, n_pages - at, n_pages), shares


def fork_and_compare(F, ctx, pt, shares, o, os, parent, keep):
    b = len(o.table)
    copies, n = torch.full((b + 2, 3), -9, dtype=torch.int32, device="cuda"), torch.full((3,), -9, dtype=torch.int32, device="cuda")
    F.flux_page_fork(ctx, pt, shares, None if parent is None else i32(parent), None if keep is None else i32(keep), copies[1:], n[1:])
    want, short = S.fork(o, os, parent, keep)
    same_pages(pt, o)
    assert shares.tolist() == os
    assert n.tolist() == [-9, len(want), -9]
    assert copies.tolist() == [[-9] * 3] + [list(x) for x in want] + [[-9] * 3] * (b + 1 - len(want))
    assert F.flux_last_device_status(ctx) == (F.FLUX_DEV_KV_OVERFLOW if short else 0)
    return want


MANY = [(3, [200 + 7 * i for i in range(5)]), (0, [0, 1, 64, 63]), (2, [128, 128, 191]), (1, [64, 500])]


@pytest.mark.parametrize("groups,parent,keep,n_pages", [
    ([(0, [0])], [0], [0], 1),
    ([(0, [1])], [-1], None, 1),
    ([(0, [100, 5])], [0, 0], None, 4),
    ([(0, [100, 64, 30])], [1, 1, 1], [64, 10, 20], 8),       # one has all of the page: both others copy it
    ([(0, [100, 64, 30])], [2, 2, -1], [9, 30, 5], 8),        # the first goes on in it
    ([(0, [100, 64, 30])], [2, 0, 1], None, 8),               # they change places
    (MANY, None, None, 64),
    (MANY, None, [0] * 14, 64),
    (MANY, [0, 0, 0, 3, 3, 8, 8, 8, -1, 9, 9, -1, 13, 13], [1000] * 14, 64),
    (MANY, [4, 4, 4, 4, 4, 0, 0, 13, 13, 13, 13, 13, 13, 12], [130, 190, 64, 1, 1000, 5, -3, 500, 499, 448, 450, 20, 0, 64], 64),
])
def test_fork(F, ctx, groups, parent, keep, n_pages):
    pt, shares, o, os = state(F, groups, 9, n_pages, len(groups))
    fork_and_compare(F, ctx, pt, shares, o, os, parent, keep)
    # what came of it is forked, cut and given back
    b = len(o.table)
    fork_and_compare(F, ctx, pt, shares, o, os, [(i * 5) % b for i in range(b)], [n - 1 for n in o.kv_len])
    fork_and_compare(F, ctx, pt, shares, o, os, [-1 if i % 3 == 0 else i for i in range(b)], None)
    fork_and_compare(F, ctx, pt, shares, o, os, None, [0] * b)
    assert o.n_free == n_pages and not any(os)


@pytest.mark.parametrize("b,wide,n_pages", [(64, 40, 3000), (300, 7, 4096), (257, 300, 40000), (1025, 4, 9000), (4096, 3, 20000), (1, 1500, 4097)])
def test_fork_at_random(F, ctx, b, wide, n_pages):
    rng = np.random.default_rng(b)
    groups, left = [], b
    while left > 0:
        m = min(left, int(rng.integers(1, 9)))
        shared = int(rng.integers(0, wide))
        groups.append((shared, [int(x) for x in rng.integers(64 * shared, 64 * min(wide, shared + max(1, n_pages // (2 * b))) + 1, m)]))
        left -= m
    pt, shares, o, os = state(F, groups, wide, n_pages, b)
    for turn in range(3):
        parent = [int(x) if x >= -b // 10 else -1 for x in rng.integers(-b // 10, b, b)]
        parent = [max(p, -1) for p in parent]
        keep = [int(x) for x in rng.integers(0, 64 * wide + 1, b)]
        keep = [k - k % 64 if rng.random() < 0.3 else k for k in keep]
        fork_and_compare(F, ctx, pt, shares, o, os, parent, keep if turn else None)
    fork_and_compare(F, ctx, pt, shares, o, os, [-1] * b, None)
    assert not any(os) and o.n_free == n_pages


def test_fork_where_pages_run_out(F, ctx):
    pt, shares, o, os = state(F, [(1, [100, 90, 128]), (0, [70])], 3, 7, 3)
    fork_and_compare(F, ctx, pt, shares, o, os, [0, 0, 0, 0], [100, 99, 98, 64])          # two pages go back, two are taken
    fork_and_compare(F, ctx, pt, shares, o, os, [0, 0, 0, 0], None)                       # one more
    pt, shares, o, os = state(F, [(0, [10]), (0, [0, 0, 0])], 2, 2, 4)
    fork_and_compare(F, ctx, pt, shares, o, os, [0, 0, 0, 0], None)                       # three are needed, one is there
    assert o.kv_len == [10, 10, 0, 0]


def test_fork_with_numbers_that_do_not_fit(F, ctx):
    """Parents, lengths, entries and lists that no program should hand over: nothing outside the buffers is touched, and the status says so."""
    copies, n = torch.full((4, 3), -9, dtype=torch.int32, device="cuda"), i32([-9])
    pt, shares, o, _ = state(F, [(0, [10, 70, 64, 5])], 4, 16, 5)
    F.flux_page_fork(ctx, pt, shares, i32([0, 7, -9, 3]), None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    assert pt.kv_len.tolist() == [10, 0, 0, 5] and n.tolist() == [0] and int(pt.n_free) == 14
    pt, shares, o, _ = state(F, [(0, [10, 70, 64, 5])], 4, 16, 5)
    pt.kv_len[1], pt.kv_len[3] = 100000, -5                  # cut to the table's 256, of which two entries are -1; and to 0
    F.flux_page_fork(ctx, pt, shares, None, None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH | F.FLUX_DEV_BAD_PAGE
    assert pt.kv_len.tolist() == [10, 256, 64, 0] and not shares.any() and n.tolist() == [0]
    pt, shares, o, _ = state(F, [(0, [10, 70, 64, 5])], 4, 16, 5)
    pt.table[1, 1] = 16
    first, free = int(pt.table[1, 0]), int(pt.n_free)
    F.flux_page_fork(ctx, pt, shares, i32([0, 2, 1, 1]), None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    assert pt.table[2].tolist() == [first, -1, -1, -1] and pt.table[3].tolist() == [first, -1, -1, -1] and pt.kv_len.tolist() == [10, 64, 70, 70]
    assert int(shares[first]) == 1 and n.tolist() == [0] and int(pt.n_free) == free + 1   # the page of sequence 3
    # a list of free pages that says too much, and a page that was shared by less than have it
    pt, shares, o, _ = state(F, [(0, [10, 10, 10, 5])], 4, 16, 5)
    pt.n_free[0] = 99
    pt.free_pages[:] = -3
    F.flux_page_fork(ctx, pt, shares, i32([0, 0, -1, 3]), None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH | F.FLUX_DEV_BAD_PAGE
    assert copies[0].tolist() == [-1, -1, 10] and int(pt.table[1, 0]) == -1 and int(pt.n_free) == 15
    pt, shares, o, _ = state(F, [(1, [64, 64, 64, 64])], 4, 16, 5)
    page = int(pt.table[0, 0])
    shares[page] = 1
    F.flux_page_fork(ctx, pt, shares, i32([-1, -1, -1, -1]), None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    assert not shares.any() and int(pt.n_free) == 16 and pt.free_pages.tolist()[15] == page


# ---- compaction and copies -------------------------------------------------------------------------------------------

def compact_and_compare(F, ctx, pt, shares, o, os, most):
    moves, n = torch.full((most + 2, 3), -9, dtype=torch.int32, device="cuda"), torch.full((3,), -9, dtype=torch.int32, device="cuda")
    F.flux_page_compact(ctx, pt, shares, moves[1:], n[1:], most)
    want = S.compact(o, os, most)
    same_pages(pt, o)
    assert shares is None or shares.tolist() == os
    assert n.tolist() == [-9, len(want), -9]
    assert moves.tolist() == [[-9] * 3] + [list(x) for x in want] + [[-9] * 3] * (most + 1 - len(want))
    assert F.flux_last_device_status(ctx) == 0
    return want


@pytest.mark.parametrize("groups,n_pages", [
    ([(0, [0])], 1), ([(0, [1])], 1), ([(0, [1])], 2), ([(0, [64])], 64), ([(0, [64])], 65), (MANY, 40), (MANY, 127), (MANY, 5000), ([(0, [64 * 30])] * 3, 90),
    ([(2, [64 * (i % 5 + 2) for i in range(6)])] * 50, 3001),
])
@pytest.mark.parametrize("most", [1, 5, 4000])
def test_compact(F, ctx, groups, n_pages, most):
    pt, shares, o, os = state(F, groups, 30, n_pages, n_pages)
    for _ in range(2):
        compact_and_compare(F, ctx, pt, shares, o, os, most)
    if most == 4000:
        assert sorted({p for row in o.table for p in row if p >= 0}) == list(range(n_pages - o.n_free))
        assert compact_and_compare(F, ctx, pt, None, o, None, 3) == []


def test_compact_of_a_large_pool(F, ctx):
    """The most pages that a call takes; 4096 sequences."""
    n_pages = 1 << 20
    pt, _, o, _ = state(F, [(0, [64 * (i % 40)]) for i in range(4096)], 40, n_pages, 1)
    moves, n = torch.full((50000, 3), -9, dtype=torch.int32, device="cuda"), i32([0])
    before = {b: list(row) for b, row in enumerate(o.table)}
    F.flux_page_compact(ctx, pt, None, moves, n, 50000)
    used = n_pages - o.n_free
    free, held = sorted(o.free[:o.n_free]), sorted(set(range(n_pages)) - set(o.free[:o.n_free]), reverse=True)
    want = [(u, f) for u, f in zip(held, free) if u > f][:50000]
    m = int(n)
    assert m == len(want) and moves[:m].tolist() == [[u, f, 64] for u, f in want] and bool((moves[m:] == -9).all())
    to = dict(want)
    assert pt.table.tolist() == [[to.get(p, p) for p in before[b]] for b in range(4096)]
    left = np.ones(n_pages, dtype=bool)
    left[[to.get(p, p) for p in held]] = False
    assert np.array_equal(pt.free_pages.cpu().numpy()[:o.n_free], np.flatnonzero(left)[::-1])
    assert int(pt.n_free) == o.n_free and used == len(held) and F.flux_last_device_status(ctx) == 0


def test_compact_with_numbers_that_do_not_fit(F, ctx):
    moves, n = torch.full((16, 3), -9, dtype=torch.int32, device="cuda"), i32([-9])
    pt, _, o, _ = state(F, [(0, [10, 70])], 4, 16, 5)
    pt.free_pages[0], pt.free_pages[1], pt.free_pages[2] = -1, 16, pt.free_pages[3]      # three entries that say nothing
    pt.table[1, 1] = 99
    F.flux_page_compact(ctx, pt, None, moves, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    assert int(pt.n_free) == 10 and int(pt.table[1, 1]) == 99
    free = pt.free_pages.tolist()[:10]
    assert free == list(range(15, 5, -1)) and all(0 <= int(pt.table[b, 0]) < 6 for b in (0, 1))
    pt, _, o, _ = state(F, [(0, [10, 70])], 4, 16, 5)
    pt.kv_len[0], pt.n_free[0] = 1 << 30, -4
    F.flux_page_compact(ctx, pt, None, moves, n)
    assert F.flux_last_device_status(ctx) & F.FLUX_DEV_BAD_LENGTH and n.tolist() == [0] and int(pt.n_free) == 0


@pytest.mark.parametrize("hkv,d,strided", [(1, 64, False), (3, 64, True), (8, 128, False), (2, 128, True)])
def test_copy(F, ctx, hkv, d, strided):
    n = 12
    codes = torch.randint(0, 256, (2, n, hkv, 64, d), dtype=torch.uint8, device="cuda")
    if strided:                                              # [page, token, head, d] with room between the pages
        store = torch.zeros(2, n, 65, hkv, d, dtype=torch.uint8, device="cuda")
        store[:, :, :64] = codes.transpose(2, 3)
        k, v = (store[i, :, :64].transpose(1, 2) for i in (0, 1))
    else:
        k, v = codes[0].clone(), codes[1].clone()
    scale = torch.rand(2, n, hkv, device="cuda")
    kv = F.PagedKV(k, v, scale[0].clone(), scale[1].clone())
    entries = [(0, 11, 64), (3, 2, 1), (-1, -1, 64), (5, 6, 63), (0, 7, 0), (9, 10, 90), (0, 1, -4), (4, 8, 17)]
    want = [codes[i].cpu().numpy().copy() for i in (0, 1)], [scale[i].cpu().numpy().copy() for i in (0, 1)]
    count = i32([len(entries) - 1])
    listed = i32([list(e) for e in entries])
    F.flux_page_copy(ctx, kv, hkv, d, listed, count)
    done = [(s, t, max(0, min(64, r))) for s, t, r in entries[:-1] if s >= 0]
    for c, s in zip(*want):
        S.copy_pages(c, s, done)
    assert np.array_equal(k.cpu().numpy(), want[0][0]) and np.array_equal(v.cpu().numpy(), want[0][1])
    assert np.array_equal(kv.k_scale.cpu().numpy(), want[1][0]) and np.array_equal(kv.v_scale.cpu().numpy(), want[1][1])
    F.flux_page_copy(ctx, kv, hkv, d, listed, None, 8)       # all of them
    for c, s in zip(*want):
        S.copy_pages(c, s, [(4, 8, 17)])
    assert np.array_equal(k.cpu().numpy(), want[0][0]) and np.array_equal(v.cpu().numpy(), want[0][1])
    assert F.flux_last_device_status(ctx) == 0
    F.flux_page_copy(ctx, kv, hkv, d, i32([[n, 1, 64], [2, -3, 64], [-1, 3, 64]]), None)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    assert np.array_equal(k.cpu().numpy(), want[0][0])
    if strided:
        assert not store[:, :, 64:].any()


# ---- together --------------------------------------------------------------------------------------------------------

def test_prompts_beams_and_compaction_together(F, ctx):
    """Prompts are appended, every sequence goes on as copies, each copy with tokens of its own, some are dropped, the pool is closed: what the
    sequences attend to is what a list of their own rows says, step by step."""
    hq, hkv, d, b, n_pages, wide = 8, 2, 64, 6, 60, 12
    (wq, wk), (_, wkx) = weights(1, d)
    f, fx = freqs(d)
    hc = F.head_cfg(hq, hkv, d, wq, wk, 1e-6, f)
    cfg = F.attn_cfg(hq, hkv, d, 4, 64, 0.0, 1)
    pt = F.PageTable.empty(b, n_pages, wide)
    kv = F.PagedKV.empty(n_pages, hkv, d)
    for x in (kv.k, kv.v):
        x.view(torch.uint8).fill_(0x7F)                      # pages that nobody wrote hold NaN
    shares, list_, n = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.empty(n_pages, 3, dtype=torch.int32, device="cuda"), i32([0])
    mode = torch.ones(b, dtype=torch.uint8, device="cuda")
    held = [[] for _ in range(b)]                            # the rows (key, value) of every sequence

    def step(new, seed):
        t = sum(new)
        slots = torch.empty(t, dtype=torch.int32, device="cuda")
        pos = [len(h) + i for h, m in zip(held, new) for i in range(m)]
        F.flux_page_plan(ctx, pt, cu_of(new), t, slots)
        _, _, (q, k, v), (_, kx, vx) = rows(seed, t, hq, hkv, d)
        qo = torch.empty(t, hq, d, dtype=torch.bfloat16, device="cuda")
        F.flux_qkv_append_paged(ctx, hc, kv, q, k, v, slots, i32(pos), t, qo)
        keys = S.heads(kx, wkx, 1e-6, pos, fx, False)
        at = 0
        for i, m in enumerate(new):
            held[i] = held[i] + [(keys[at + j], vx[at + j]) for j in range(m)]
            at += m
        out = torch.empty(t, hq, d, device="cuda")
        F.flux_attn_prefill_paged(ctx, cfg, qo, cu_of(new), max(new), 64 * wide, kv, pt, mode, out)
        at = 0
        for i, m in enumerate(new):
            if m:
                kh, vh = np.stack([r[0] for r in held[i]]), np.stack([r[1] for r in held[i]])
                ref = O.attention(qo[at:at + m].double().cpu().numpy(), kh, vh, 1, 4, 64)
                # codes of keys and values are off by 2^-4 of a value at most and weigh each other out over many keys; a row of
                # somebody else's moves a result by much more
                off = np.abs(out[at:at + m].double().cpu().numpy() - ref)
                assert off.max() < 0.25 and np.sqrt((off ** 2).mean()) < 0.04, (i, off.max())
            at += m

    def fork(parent, keep):
        F.flux_page_fork(ctx, pt, shares, i32(parent), i32(keep), list_, n)
        F.flux_page_copy(ctx, kv, hkv, d, list_, n)
        held[:] = [held[p][:k] if p >= 0 else [] for p, k in zip(parent, keep)]
        assert pt.kv_len.tolist() == [len(h) for h in held]

    step([150, 0, 0, 200, 0, 0], 1)
    fork([0, 0, 0, 3, 3, 3], [999] * 6)
    assert int((shares > 0).sum()) == 2 + 3 and int(n) == 4
    step([1, 2, 3, 70, 1, 1], 2)
    step([1] * 6, 3)
    fork([1, 1, 0, 3, 3, -1], [150, 152, 999, 230, 192, 0])
    step([5, 1, 1, 1, 64, 0], 4)
    F.flux_page_compact(ctx, pt, shares, list_, n)
    F.flux_page_copy(ctx, kv, hkv, d, list_, n)
    used = n_pages - int(pt.n_free)
    assert int(pt.table.max()) < used
    step([1, 1, 1, 1, 1, 90], 5)
    fork([-1] * 6, [0] * 6)
    assert int(pt.n_free) == n_pages and not shares.any() and F.flux_last_device_status(ctx) == 0


def test_captured_forks_are_replayed(F, ctx):
    """A scheduling step (fork, copies, plan, append) in a graph, replayed with other parents and eager calls between the replays."""
    hq, hkv, d, b, wide, n_pages = 4, 2, 64, 8, 6, 64
    groups = [(1, [100, 90, 130, 64]), (2, [130, 140, 150, 190])]
    pt, shares, o, os = state(F, groups, wide, n_pages, 9)
    codes = torch.randint(0, 0x7F, (2, n_pages, hkv, 64, d), dtype=torch.uint8, device="cuda")
    kv = F.PagedKV(codes[0], codes[1], *(torch.full((n_pages, hkv), 2.0 ** -7, device="cuda") for _ in range(2)))
    ref = [c.cpu().numpy().copy() for c in codes], [np.full((n_pages, hkv), 2.0 ** -7, dtype=np.float32) for _ in range(2)]
    parent, keep, copies, n = i32([0] * b), i32([0] * b), torch.empty(b, 3, dtype=torch.int32, device="cuda"), i32([0])
    cu, slots = cu_of([1] * b), torch.empty(b, dtype=torch.int32, device="cuda")
    _, _, (_, k, v), _ = rows(3, b, hq, hkv, d)
    kx, vx = k.double().cpu().numpy(), v.double().cpu().numpy()

    def calls():
        F.flux_page_fork(ctx, pt, shares, parent, keep, copies, n)
        F.flux_page_copy(ctx, kv, hkv, d, copies, n)
        F.flux_page_plan(ctx, pt, cu, b, slots)
        F.flux_qkv_append_paged(ctx, F.head_cfg(hq, hkv, d), kv, None, k, v, slots, None, b, None)

    graph = torch.cuda.CUDAGraph()
    before = [x.clone() for x in (pt.table, pt.kv_len, pt.free_pages, pt.n_free, shares, codes, kv.k_scale, kv.v_scale)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()                                              # (warm, then everything as it was)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip((pt.table, pt.kv_len, pt.free_pages, pt.n_free, shares, codes, kv.k_scale, kv.v_scale), before):
        x.copy_(y)
    with torch.cuda.graph(graph):
        calls()
    rng = np.random.default_rng(4)
    for turn in range(5):
        p = [int(x) for x in rng.integers(-1, b, b)]
        m = [int(x) for x in rng.integers(0, 300, b)]
        parent.copy_(i32(p)), keep.copy_(i32(m))
        if turn % 2 == 0:
            graph.replay()
        else:
            calls()
        torch.cuda.synchronize()
        entries, short = S.fork(o, os, p, m)
        planned, over = o.plan([1] * b)
        assert not short and not over and slots.tolist() == planned
        same_pages(pt, o)
        assert shares.tolist() == os
        for c, s, y in zip(*ref, (kx, vx)):
            S.copy_pages(c, s, entries)
            P.append(c, s, y, planned)
        assert np.array_equal(codes.cpu().numpy(), np.stack(ref[0])) and np.array_equal(kv.k_scale.cpu().numpy(), ref[1][0])
    assert F.flux_last_device_status(ctx) == 0
