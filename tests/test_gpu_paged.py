"""The paged 8-bit KV cache on the GPU: page planning and release, the quantising append, decode attention over pages, against
their plain definitions (oracle/paged_oracle.py and the float64 attention oracle)."""
import numpy as np
import pytest
import torch

from oracle import flux_oracle as O
from oracle import paged_oracle as P
from tests import helpers as H

pytestmark = pytest.mark.gpu

FA, SA = 1, 0


@pytest.fixture(scope="module")
def F():
    from paper_2604_07394_amd import binding
    return binding


@pytest.fixture()
def ctx(F):
    c = F.flux_create(0, 0)
    yield c
    torch.cuda.synchronize()
    F.flux_destroy(c)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def cu_of(rows):
    return i32(np.concatenate([[0], np.cumsum(rows)]))


def bf16(x):
    """float64 values rounded to bf16: the device tensor, and the values it holds."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


# ---- pages -----------------------------------------------------------------------------------------------------------

def page_state(F, lens, table_pages, n_pages, seed, used=None):
    """Tables of sequences with `lens` cached tokens on shuffled pages; the rest is free (or `used` of it)."""
    ids = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((len(lens), table_pages), -1)
    at = 0
    for b, n in enumerate(lens):
        k = -(-n // 64)
        table[b, :k] = ids[at:at + k]
        at += k
    free = np.full(n_pages, -7)
    free[:n_pages - at] = ids[at:]
    n_free = n_pages - at if used is None else used
    return F.PageTable(i32(table), i32(lens), i32(free), i32([n_free])), P.Pages(table, lens, free, n_free, n_pages)


def same_pages(pt, o):
    assert pt.table.tolist() == o.table and pt.kv_len.tolist() == o.kv_len
    assert pt.free_pages.tolist() == o.free and pt.n_free.tolist() == [o.n_free]


@pytest.mark.parametrize("lens,rows,table_pages,n_pages", [
    ([0], [1], 1, 1),
    ([0], [64], 2, 3),
    ([63, 64, 65, 0, 128], [1, 1, 1, 0, 0], 4, 12),
    ([5, 0, 700], [59, 130, 1000], 30, 64),
    ([10] * 300, [1] * 300, 3, 400),
    ([64] * 257, [1] * 257, 3, 600),
    ([0] * 3, [5000, 1, 2100], 90, 200),                     # several workgroups of slots
    ([i % 130 for i in range(4096)], [(i * 7) % 3 for i in range(4096)], 4, 20000),
])
def test_plan_and_release(F, ctx, lens, rows, table_pages, n_pages):
    pt, o = page_state(F, lens, table_pages, n_pages, len(lens))
    t = sum(rows)
    slots = torch.full((t + 8,), -9, dtype=torch.int32, device="cuda")
    F.flux_page_plan(ctx, pt, cu_of(rows), t, slots)
    want, overflow = o.plan(rows)
    assert not overflow and slots.tolist() == want + [-9] * 8
    same_pages(pt, o)
    keep = [n if b % 3 == 0 else (0 if b % 3 == 1 else n + rows[b] - 1) for b, n in enumerate(lens)]
    F.flux_page_release(ctx, pt, i32(keep))
    o.release(keep)
    same_pages(pt, o)
    # what was taken back is planned again as before
    rows2 = [a + b - c for a, b, c in zip(lens, rows, o.kv_len)]
    F.flux_page_plan(ctx, pt, cu_of(rows2), sum(rows2), slots)
    o.plan(rows2)
    same_pages(pt, o)
    assert F.flux_last_device_status(ctx) == 0


def test_plan_where_pages_or_table_rows_run_out(F, ctx):
    pt, o = page_state(F, [60, 0, 10, 64], 3, 9, 3, used=3)
    rows = [200, 65, 40, 20]                                 # sequence 0: its table row is full at 192; then two free pages, then none
    slots = torch.empty(sum(rows), dtype=torch.int32, device="cuda")
    F.flux_page_plan(ctx, pt, cu_of(rows), sum(rows), slots)
    want, overflow = o.plan(rows)
    assert overflow and slots.tolist() == want and -1 in want
    same_pages(pt, o)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_KV_OVERFLOW
    F.flux_page_plan(ctx, pt, cu_of(rows), 0, slots)         # nothing to do
    same_pages(pt, o)


def test_plan_with_numbers_that_do_not_fit(F, ctx):
    """Lengths, prefix sums and page numbers that no program should hand over: nothing outside the buffers is touched, and the
    status says so."""
    pt, _ = page_state(F, [10, 70, 0, 5], 4, 16, 5)
    pt.table[0, 0] = 16                                      # the partly filled page of sequence 0 is not in the pool
    pt.free_pages[int(pt.n_free) - 1] = -3                   # ... nor is the first free page
    guard = torch.full((64,), -9, dtype=torch.int32, device="cuda")
    slots = guard[8:24]
    F.flux_page_plan(ctx, pt, i32([0, 2, 4, 6, 8]), 8, slots)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE | F.FLUX_DEV_KV_OVERFLOW
    got = slots.tolist()
    assert got[:2] == [-1, -1] and got[2] == int(pt.table[1, 1]) * 64 + 6 and got[4:6] == [-1, -1] and got[8:] == [-9] * 8
    assert int(pt.table[2, 0]) == -1 and pt.kv_len.tolist() == [10, 72, 2, 7]
    # lengths and sums
    pt, _ = page_state(F, [10, 70, 0, 5], 4, 16, 5)
    pt.kv_len[1], pt.kv_len[3] = 1000, -4
    F.flux_page_plan(ctx, pt, i32([0, 3, 1, 90, 8]), 8, slots)
    assert F.flux_last_device_status(ctx) & F.FLUX_DEV_BAD_LENGTH
    assert pt.kv_len[1] == 256 and pt.kv_len[3] == 0 and (guard[:8] == -9).all() and (guard[24:] == -9).all()
    pt, _ = page_state(F, [10, 70, 0, 5], 4, 16, 5)
    pt.n_free[0] = 99
    pt.free_pages[:] = -1
    F.flux_page_plan(ctx, pt, i32([0, 0, 0, 4, 4]), 4, slots)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH | F.FLUX_DEV_BAD_PAGE
    # release: entries outside the pool are not listed, nor is anything past n_pages
    pt, _ = page_state(F, [130, 64], 4, 5, 6)
    pt.table[0, 1] = 77
    before = pt.free_pages.tolist()
    first, last, other = int(pt.table[0, 0]), int(pt.table[0, 2]), int(pt.table[1, 0])
    F.flux_page_release(ctx, pt, i32([0, 0]))
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    assert pt.n_free.tolist() == [4] and pt.free_pages.tolist() == before[:1] + [other, last, first] + before[4:]
    assert (pt.table == -1).all() and pt.kv_len.tolist() == [0, 0]
    pt, _ = page_state(F, [130, 64], 4, 5, 6)
    pt.n_free[0] = 3
    F.flux_page_release(ctx, pt, i32([0, -5]))
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE and pt.n_free.tolist() == [5]


# ---- append ----------------------------------------------------------------------------------------------------------

def pool_of(n_pages, hkv, d, seed=0, fill=None):
    """Random codes and scales of K and V as NumPy arrays."""
    rng = np.random.default_rng(seed)
    codes = [rng.integers(0, 256, (n_pages, hkv, 64, d), dtype=np.uint8) if fill is None else np.full((n_pages, hkv, 64, d), fill, np.uint8) for _ in range(2)]
    scale = [np.ldexp(1.0, rng.integers(-9, -5, (n_pages, hkv))).astype(np.float32) for _ in range(2)]
    return codes, scale


def paged_kv(F, codes, scale, layout="phtd"):
    def dev(x):
        n, h, _, d = x.shape
        if layout == "phtd":
            t = torch.empty(n, h, 64, d, dtype=torch.uint8, device="cuda")
        elif layout == "pthd":                               # a token's heads next to each other
            t = torch.empty(n, 64, h, d, dtype=torch.uint8, device="cuda").transpose(1, 2)
        else:                                                # rows with room between them
            t = torch.empty(n, h, 64, d + 48, dtype=torch.uint8, device="cuda")[..., 16:16 + d]
        t.copy_(torch.from_numpy(x))
        return t
    return F.PagedKV(dev(codes[0]), dev(codes[1]), torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda())


def same_pool(kv, codes, scale):
    for t, x in ((kv.k, codes[0]), (kv.v, codes[1])):
        got = t.cpu().numpy()
        nan = (x & 0x7F) == 0x7F                             # (either sign)
        assert np.array_equal(nan, (got & 0x7F) == 0x7F)
        assert np.array_equal(got[~nan], x[~nan])
    assert np.array_equal(kv.k_scale.cpu().numpy(), scale[0]) and np.array_equal(kv.v_scale.cpu().numpy(), scale[1])


def slots_behind(cached, rows, n_pages, seed):
    ids = np.random.default_rng(seed).permutation(n_pages)
    slots, at = [], 0
    for c, n in zip(cached, rows):
        held = -(-(c + n) // 64)
        slots += [int(ids[at + p // 64]) * 64 + p % 64 for p in range(c, c + n)]
        at += held
    assert at <= n_pages
    return slots


@pytest.mark.parametrize("cached,rows,hkv,d,layout", [
    ([0], [1], 1, 64, "phtd"),
    ([63], [1], 2, 128, "phtd"),
    ([0, 64, 5], [64, 64, 59], 2, 128, "pthd"),
    ([1, 62, 0, 33], [1, 1, 1, 1], 3, 64, "wide"),
    ([17, 0, 63, 40], [200, 1, 66, 3], 4, 128, "phtd"),
    ([9] * 40, [1 + i % 5 for i in range(40)], 8, 64, "pthd"),
    ([3, 0, 31], [3000, 1000, 333], 5, 128, "phtd"),         # more rows than a wave each
    ([3, 0, 31, 64], [2000, 1100, 333, 1], 8, 64, "wide"),
])
def test_append_quantises_bit_for_bit(F, ctx, cached, rows, hkv, d, layout):
    rng = np.random.default_rng(sum(cached) + d)
    n_pages = sum(-(-(c + n) // 64) for c, n in zip(cached, rows)) + 2
    codes, scale = pool_of(n_pages, hkv, d, seed=d)
    for x in codes:                                          # the rows that pages hold are finite
        x[(x & 0x7F) == 0x7F] = 5
    kv = paged_kv(F, codes, scale, layout)
    slots = slots_behind(cached, rows, n_pages, hkv)
    for i in range(len(rows), 0, -1):                        # rows without a place stand behind those of their sequence
        slots[sum(rows[:i]):sum(rows[:i])] = [-1] * (i % 4)
    t = len(slots)
    # magnitudes of every size: blocks whose scale grows, shrinks or stays, tiny and zero rows
    k, kf = bf16(rng.standard_normal((t, hkv, d)) * 2.0 ** rng.integers(-6, 6, (t, hkv, 1)))
    v, vf = bf16(rng.standard_normal((t, hkv, d)) * 2.0 ** (rng.integers(-3, 3, (t, 1, 1)) * 20.0) * (rng.random((t, hkv, 1)) > 0.2))
    F.flux_kv_append_paged(ctx, kv, hkv, d, k, v, i32(slots), t)
    P.append(codes[0], scale[0], kf, slots)
    P.append(codes[1], scale[1], vf, slots)
    same_pool(kv, codes, scale)
    assert F.flux_last_device_status(ctx) == 0


@pytest.mark.parametrize("t,hkv", [(70, 2), (9000, 4)])      # either instance
def test_append_of_values_that_are_not_finite_and_slots_that_do_not_exist(F, ctx, t, hkv):
    d, n_pages = 64, -(-t // 64)
    codes, scale = pool_of(n_pages, hkv, d, 3, fill=0)
    kv = paged_kv(F, codes, scale)
    rng = np.random.default_rng(2)
    x = rng.standard_normal((t, hkv, d))
    x[5, 0, 3], x[6, 1, 0], x[66, 0, 63], x[7, 0, 1] = np.inf, -np.inf, np.nan, 3e38
    k, kf = bf16(x)
    slots = list(range(t))
    slots[64:70] = [n_pages * 64, n_pages * 64 + 1, 2 ** 31 - 1, 2 ** 31 - 64, -1, -2 ** 31]
    F.flux_kv_append_paged(ctx, kv, hkv, d, k, k, i32(slots), t)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    kept = [s if 0 <= s < n_pages * 64 else -1 for s in slots]
    P.append(codes[0], scale[0], kf, kept)
    P.append(codes[1], scale[1], kf, kept)
    same_pool(kv, codes, scale)


# ---- decode ----------------------------------------------------------------------------------------------------------

def attention_case(F, lens, hq, hkv, d, layout="phtd", seed=0, rows=None, table_pages=None, spare=3):
    """A pool with the sequences' pages scattered over it, and what their positions stand for.  Everything that no sequence
    attends to holds NaN: codes behind the lengths, spare pages, and the table points outside the pool behind its end."""
    rng = np.random.default_rng(seed)
    held = [-(-n // 64) for n in lens]
    n_pages = sum(held) + spare
    ids = rng.permutation(n_pages)
    codes = [torch.from_numpy(rng.standard_normal((n_pages, hkv, 64, d)) * 2.0).to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy() for _ in range(2)]
    scale = [rng.uniform(0.2, 0.8, (n_pages, hkv)).astype(np.float32) for _ in range(2)]
    wide = table_pages or max(held) + 2
    table = np.where(np.arange(wide) % 2 == 0, 2 ** 30, -5)[None].repeat(len(lens), 0)
    seqs, at = [], 0
    for b, n in enumerate(lens):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
        seqs.append([P.gather(c, s, table[b], n) for c, s in zip(codes, scale)])
        if n % 64:
            for c in codes:
                c[table[b, held[b] - 1], :, n % 64:] = 0x7F
    for c, s in zip(codes, scale):
        c[ids[at:]] = 0xFF
        s[ids[at:]] = np.nan
    q, qf = bf16(rng.standard_normal((len(lens) if rows is None else sum(rows), hq, d)))
    pt = F.PageTable(i32(table), i32(lens), i32([0] * n_pages), i32([0]))
    return paged_kv(F, codes, scale, layout), pt, q, qf, seqs


def tolerance(qf, seqs, d, scale=None):
    """What the fp32 arithmetic may be off by, in units of the largest |v|.  A weight is off by 2^-16 (two bf16 terms) and by twice the
    error of its score, which sums d exact products in fp32: at most (d + 4) 2^-24 of |q| |k| scale each way."""
    k = max(float(np.sqrt((s[0] ** 2).sum(-1)).max()) if s[0].size else 0.0 for s in seqs)
    s = float(np.sqrt((qf ** 2).sum(-1)).max()) * k * (d ** -0.5 if scale is None else scale)
    return 2 * (2.0 ** -16 + 2 * (d + 4) * 2.0 ** -24 * s)


def check(out, ref, eps, seqs):
    got = H.torch_to_f64(out)
    assert np.isfinite(got).all()
    v = max(float(np.abs(s[1]).max()) if s[1].size else 0.0 for s in seqs)
    bound = eps * v + (2.0 ** -8 * np.abs(ref) if out.dtype == torch.bfloat16 else 0)
    worst = np.abs(got - ref) - bound
    assert (worst <= 0).all(), (float(np.abs(got - ref).max()), eps * v)
    # roundings are independent, so that their sum is far below the bound: 4e-5 of the 2-norm (bf16 output: half a step of 2^-8, 2^-9 on average at most)
    rel = np.sqrt(((got - ref) ** 2).sum() / max((ref ** 2).sum(), 1e-300))
    assert rel <= (4e-5 if out.dtype == torch.float32 else 4e-5 + 2.0 ** -9 * 2), rel


def decode_ref(qf, seqs, modes, n_sink, window, block=1, scale=None):
    out = np.zeros(qf.shape)
    for b, (k, v) in enumerate(seqs):
        if len(k):
            out[b] = O.attention(qf[b][None], k, v, modes[b], n_sink, window, scale, block=block)[0]
    return out


CASES = [
    # lens, modes, hq, hkv, d, n_sink, window, sa_block
    ([1], [FA], 1, 1, 64, 0, 1, 0),
    ([0, 1, 63, 64, 65, 127, 128, 129], [FA] * 8, 4, 2, 128, 4, 16, 0),
    ([0, 1, 63, 64, 65, 127, 128, 129, 200, 1000], [SA] * 10, 4, 2, 64, 4, 16, 0),
    ([700, 300, 64, 1500], [SA, FA, SA, SA], 8, 2, 128, 16, 128, 0),
    ([700, 300, 64, 1500], [SA, FA, SA, SA], 8, 2, 128, 16, 128, 64),
    ([700, 301, 64, 1500], [SA, SA, FA, SA], 14, 2, 128, 100, 130, 16),      # group 7
    ([500, 40], [SA, FA], 40, 2, 64, 0, 1, 0),                               # group 20: two blocks of queries; a window of one
    ([3000], [SA], 16, 1, 128, 64, 64, 0),                                   # group 16; whole pages of sinks and window
    ([5000, 9, 12000], [FA, FA, SA], 32, 8, 128, 128, 4096, 0),
    ([20000], [FA], 4, 1, 64, 0, 1, 0),
    ([20000] * 3, [FA, SA, FA], 28, 4, 128, 2 ** 31 - 1, 2 ** 31 - 1, 64),   # the sparse rule sees everything
    ([130 + 17 * (i % 23) for i in range(70)], [i % 2 for i in range(70)], 8, 8, 64, 3, 70, 0),
    ([64 * (i % 5) for i in range(300)], [FA] * 300, 4, 2, 64, 3, 70, 0),
    ([i % 3 for i in range(2100)], [FA] * 2100, 2, 2, 64, 0, 5, 0),
]


@pytest.mark.parametrize("fp32", [1, 0])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_decode_against_the_oracle(F, ctx, case, fp32):
    lens, modes, hq, hkv, d, n_sink, window, block = case
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, ("phtd", "pthd", "wide")[len(lens) % 3], seed=len(lens) + d)
    guard = torch.full((len(lens) + 2, hq, d), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, n_sink, window, 0.0, fp32, block)
    mode = torch.tensor(modes, dtype=torch.uint8, device="cuda")
    F.flux_attn_decode_paged(ctx, cfg, q, max(lens), kv, pt, mode, guard[1:-1])
    ref = decode_ref(qf, seqs, modes, n_sink, window, max(1, block))
    check(guard[1:-1], ref, tolerance(qf, seqs, d), seqs)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    assert F.flux_last_device_status(ctx) == 0
    # the largest bound is as good, and a second call the same to the bit
    again = torch.empty_like(guard[1:-1])
    F.flux_attn_decode_paged(ctx, cfg, q, max(lens), kv, pt, mode, again)
    assert torch.equal(again, guard[1:-1])
    F.flux_attn_decode_paged(ctx, cfg, q, 64 * pt.table.shape[1], kv, pt, mode, again)
    check(again, ref, tolerance(qf, seqs, d), seqs)


def test_decode_over_more_pages_than_a_wave_looks_up_at_once(F, ctx):
    """One list of 2048 pages shared out over 8 pairs: a wave's pages are asked for 64 at a time, here more than three times."""
    lens, hq, hkv, d = [40000, 131072, 90001], 8, 8, 64
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=5)
    ws = F.flux_workspace_needed(F.attn_cfg(hq, hkv, d, 0, 1), 3, 131072)
    small = F.flux_create(0, ws)                             # the workspace that is said to be enough
    out = torch.empty(3, hq, d, dtype=torch.float32, device="cuda")
    F.flux_attn_decode_paged(small, F.attn_cfg(hq, hkv, d, 0, 1, 0.3, 1), q, 131072, kv, pt, torch.ones(3, dtype=torch.uint8, device="cuda"), out)
    ref = np.zeros(qf.shape)
    for b, (k, v) in enumerate(seqs):
        for h in range(hq):
            s = 0.3 * (k[:, h] @ qf[b, h])
            p = np.exp(s - s.max())
            ref[b, h] = p @ v[:, h] / p.sum()
    check(out, ref, tolerance(qf, seqs, d, 0.3), seqs)
    torch.cuda.synchronize()
    F.flux_destroy(small)


def test_decode_where_pages_are_missing_or_the_bound_is_too_low(F, ctx):
    hq, hkv, d = 8, 2, 128
    lens = [300, 200, 64]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=9)
    pt.table[0, 1], pt.table[0, 3], pt.table[2, 0] = -1, kv.k.shape[0], 2 ** 31 - 1
    out = torch.full((3, hq, d), 7.0, dtype=torch.float32, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1)
    mode = torch.ones(3, dtype=torch.uint8, device="cuda")
    F.flux_attn_decode_paged(ctx, cfg, q, 300, kv, pt, mode, out)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    there = np.r_[0:64, 128:192, 256:300]
    left = [[x[there] for x in seqs[0]], seqs[1], [x[:0] for x in seqs[2]]]
    ref = decode_ref(qf, left, [FA] * 3, 0, 1)
    check(out, ref, tolerance(qf, seqs, d), seqs)
    assert (out[2] == 0).all()
    # a bound of two pages: the oldest are kept
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=9)
    F.flux_attn_decode_paged(ctx, cfg, q, 128, kv, pt, mode, out)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    check(out, decode_ref(qf, [[x[:128] for x in s] for s in seqs], [FA] * 3, 0, 1), tolerance(qf, seqs, d), seqs)
    # lengths that do not fit are clamped
    pt.kv_len[0], pt.kv_len[1] = -3, 10 ** 9
    F.flux_attn_decode_paged(ctx, cfg, q, 64, kv, pt, mode, out)
    assert F.flux_last_device_status(ctx) & F.FLUX_DEV_BAD_LENGTH
    assert (out[0] == 0).all() and torch.isfinite(out).all()


def test_sequences_may_share_pages(F, ctx):
    hq, hkv, d = 8, 4, 64
    kv, pt, q, qf, seqs = attention_case(F, [200, 130], hq, hkv, d, seed=4)
    pt.table[1, :2] = pt.table[0, :2]                        # the same prefix; the second one's last two positions are its own
    shared = [np.concatenate([a[:128], b[128:]]) for a, b in zip(*seqs)]
    out = torch.empty(2, hq, d, dtype=torch.float32, device="cuda")
    F.flux_attn_decode_paged(ctx, F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1), q, 200, kv, pt, torch.ones(2, dtype=torch.uint8, device="cuda"), out)
    check(out, decode_ref(qf, [seqs[0], shared], [FA, FA], 0, 1), tolerance(qf, seqs, d), seqs)


def test_nan_is_seen_only_by_those_who_look(F, ctx):
    """A NaN code among the visible keys of one head makes that head's row NaN; hidden by the sparse rule it is not read."""
    hq, hkv, d, lens = 4, 2, 128, [400, 400]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=8)
    for b in (0, 1):
        page = int(pt.table[b, 3])                           # positions 192 ..: hidden are 16 .. 199
        kv.k[page, 0, 3], kv.v[page, 0, 5] = 0x7F, 0xFF
    out = torch.empty(2, hq, d, dtype=torch.float32, device="cuda")
    F.flux_attn_decode_paged(ctx, F.attn_cfg(hq, hkv, d, 16, 200, 0.0, 1), q, 400, kv, pt, torch.tensor([1, 0], dtype=torch.uint8, device="cuda"), out)
    assert torch.isnan(out[0, :2]).all() and torch.isfinite(out[0, 2:]).all()
    ref = decode_ref(qf[1:], seqs[1:], [SA], 16, 200)
    check(out[1:], ref, tolerance(qf, seqs, d), seqs)


@pytest.mark.parametrize("batch,hq,hkv", [(1, 4, 2), (40, 16, 8), (300, 16, 8)])   # launches of 2, 320 and 2400 lists
@pytest.mark.parametrize("cached", [0, 70])
def test_decode_with_a_bound_of_zero(F, ctx, batch, hq, hkv, cached):
    """No page may be read then: rows of zeros, and a word of warning where there are some."""
    kv, pt, q, _, _ = attention_case(F, [cached] * batch, hq, hkv, 64, seed=batch)
    out = torch.full((batch, hq, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    F.flux_attn_decode_paged(ctx, F.attn_cfg(hq, hkv, 64, 4, 16), q, 0, kv, pt, torch.ones(batch, dtype=torch.uint8, device="cuda"), out)
    assert (out == 0).all()
    assert F.flux_last_device_status(ctx) == (F.FLUX_DEV_BAD_LENGTH if cached else 0)


@pytest.mark.parametrize("lens", [[3], [200], [2000, 64], [30000]])   # one wave, waves without a page, parts
@pytest.mark.parametrize("d", [64, 128])
def test_scores_far_below_zero(F, ctx, lens, d):
    """Scores of -2^17 d^0.5 for every key but some of twice that: the weights are relative to the largest one however low it lies,
    and the result is the mean of V over the first ones.  (q and the keys are powers of two and so are the scales: the scores are
    exact, and what the exponent's rounding leaves of a weight is the same for all keys.)"""
    hq, hkv = 4, 2
    rng = np.random.default_rng(d)
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=5)
    q.fill_(-2.0 ** 17)
    low = torch.from_numpy(rng.random(tuple(kv.k.shape[:3])) < 0.3).cuda()
    one = [int(torch.tensor([x], dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)) for x in (1.0, 2.0)]
    kv.k.copy_(torch.where(low, one[1], one[0])[..., None].expand(kv.k.shape).to(torch.uint8))
    kv.k_scale.fill_(1.0)
    kv.v_scale.copy_(torch.exp2(torch.floor(torch.log2(kv.v_scale))))
    table, codes, scale = pt.table.cpu().numpy(), kv.v.cpu().numpy(), kv.v_scale.cpu().numpy()
    seqs = [[None, P.gather(codes, scale, table[b], n)] for b, n in enumerate(lens)]
    ref = np.zeros((len(lens), hq, d))
    for b, n in enumerate(lens):
        flag = low.cpu().numpy()[table[b, :-(-n // 64)]].transpose(0, 2, 1).reshape(-1, hkv)[:n]
        for h in range(hq):
            keep = ~flag[:, h // 2] if not flag[:, h // 2].all() else flag[:, h // 2]
            ref[b, h] = seqs[b][1][keep, h // 2].mean(0)
    out = torch.empty(len(lens), hq, d, dtype=torch.float32, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1)
    mode = torch.ones(len(lens), dtype=torch.uint8, device="cuda")
    v = max(float(np.abs(s[1]).max()) for s in seqs)
    F.flux_attn_decode_paged(ctx, cfg, q, max(lens), kv, pt, mode, out)
    # all weights are alike: sums of n terms in fp32, 2^-24 of the sum of the magnitudes a term and as much for the denominator; two
    # terms leave 2^-16 of a weight
    assert np.abs(H.torch_to_f64(out) - ref).max() <= (2 * (max(lens) + 8) * 2.0 ** -24 + 2 * 2.0 ** -16) * v
    # the same as a run of one query, and as a tile (the bound on the queries says which)
    for most in (1, max(lens)):
        F.flux_attn_prefill_paged(ctx, cfg, q, cu_of([1] * len(lens)), most, max(lens), kv, pt, mode, out)
        # (the denominator sums the rounded weights)
        assert np.abs(H.torch_to_f64(out) - ref).max() <= (2 * (max(lens) + 8) * 2.0 ** -24 + 2 * 2.0 ** -16) * v
    assert F.flux_last_device_status(ctx) == 0
