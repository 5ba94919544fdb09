"""Norms and rotation of heads on the GPU, alone and on their way into the contiguous and the paged cache, against their plain
definitions in float64 (oracle/serving_oracle.py, oracle/paged_oracle.py)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from oracle import serving_oracle as S
from tests.test_gpu_paged import F, bf16, ctx, cu_of, i32  # noqa: F401

pytestmark = pytest.mark.gpu
EPS = 1e-6


def freqs(rot, base=10000.0):
    f = (base ** -(np.arange(0, rot, 2) / rot)).astype(np.float32)
    return torch.from_numpy(f).cuda(), f.astype(np.float64)


def rows(seed, t, hq, hkv, d, scale=1.0):
    """The projection's output on the device (query, key and value heads side by side), and its values."""
    dev, x = bf16(np.random.default_rng(seed).normal(size=(t, hq + 2 * hkv, d)) * scale)
    return dev, x, (dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]), (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])


def weights(seed, d, norm=True):
    if not norm:
        return (None, None), (None, None)
    a, b = (bf16(np.random.default_rng(seed + i).uniform(0.5, 1.5, d)) for i in (1, 2))
    return (a[0], b[0]), (a[1], b[1])


def near_enough(got, want, normed, rot, interleaved):
    """bf16 results of fp32 steps.  The rounding: half a step, 2^-8 of the value.  Before it: the mean of squares is 16 + 3 sums of
    terms of one sign (19 * 2^-24), its square root's reciprocal an instruction of one step (2^-23), two products (2^-23): below 2^-18 of a
    normed value; sine and cosine of a fraction of a turn that is rounded to 2^-26: 2^-23, and what the instructions leave, taken as 2^-19;
    so 2^-17 of the magnitudes that a turned value is made of.  The smallest bf16 step is 2^-133."""
    got = got.double().cpu().numpy()
    size = np.abs(normed).copy()
    for i in range(rot // 2):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        size[..., p] = size[..., q] = np.abs(normed[..., p]) + np.abs(normed[..., q])
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * size + 2.0 ** -133
    off = np.abs(got - want)
    assert (off <= tol).all(), (float((off / tol).max()), np.argwhere(off > tol)[:3])


CASES = [
    # t, hq, hkv, d, rot, interleaved, norm
    (1, 8, 2, 64, 64, 0, True),
    (1, 1, 1, 64, 16, 1, True),
    (7, 8, 2, 64, 32, 1, True),
    (5, 28, 4, 128, 128, 0, False),
    (3, 32, 8, 128, 64, 0, True),
    (4, 12, 1, 128, 112, 0, True),
    (9, 5, 3, 128, 48, 1, False),
    (6, 7, 7, 64, 0, 0, True),
    (2, 40, 10, 128, 128, 1, True),
    (2100, 6, 2, 64, 64, 0, True),
    (300, 32, 8, 128, 128, 0, True),
]


@pytest.mark.parametrize("t,hq,hkv,d,rot,near,norm", CASES)
@pytest.mark.parametrize("apart", [False, True])
def test_heads(F, ctx, t, hq, hkv, d, rot, near, norm, apart):
    """apart: the rows of the tokens lie next to each other, and a head's result goes where it came from."""
    dev, x, (q, k, _), (qx, kx, _) = rows(t, t, hq, hkv, d)
    (wq, wk), (wqx, wkx) = weights(t, d, norm)
    f, fx = freqs(rot) if rot else (None, None)
    pos = np.random.default_rng(t).integers(0, 5000, t)
    hc = F.head_cfg(hq, hkv, d, wq, wk, EPS, f, rot, near)
    if apart:
        q, k = q.contiguous(), k.contiguous()
        qo, ko = q, k
    else:
        qo, ko = (torch.full((t + 1, h, d), -7.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
    F.flux_qk_norm_rope(ctx, hc, q, k, i32(pos), t, qo, ko)
    for got, y, w in ((qo, qx, wqx), (ko, kx, wkx)):
        n = S.normed(y, w, EPS)
        near_enough(got[:t], n if not rot else S.turned(n, pos, fx, near), n, rot, near)
        assert apart or bool((got[t:] == -7.0).all())
    if not apart:
        assert torch.equal(dev, torch.from_numpy(x).to(torch.bfloat16).cuda())


def test_far_and_negative_positions(F, ctx):
    """Angles of millions of turns: what is left of them after whole turns is exact."""
    pos = [0, 1, -1, 63, 1 << 20, (1 << 24) + 1, 123456789, -(1 << 30), (1 << 31) - 1, -(1 << 31)]
    t, hq, hkv, d = len(pos), 4, 2, 64
    _, _, (q, k, _), (qx, kx, _) = rows(3, t, hq, hkv, d)
    f, fx = freqs(64)
    qo = torch.empty(t, hq, d, dtype=torch.bfloat16, device="cuda")
    ko = torch.empty(t, hkv, d, dtype=torch.bfloat16, device="cuda")
    F.flux_qk_norm_rope(ctx, F.head_cfg(hq, hkv, d, inv_freq=f), q, k, i32(pos), t, qo, ko)
    near_enough(qo, S.turned(qx, pos, fx, False), qx, 64, False)
    near_enough(ko, S.turned(kx, pos, fx, False), kx, 64, False)


def test_queries_or_keys_alone(F, ctx):
    _, _, (q, k, _), (qx, kx, _) = rows(4, 33, 6, 2, 128)
    (wq, wk), (wqx, wkx) = weights(4, 128)
    hc = F.head_cfg(6, 2, 128, wq, wk, EPS)
    qo, ko = torch.empty(33, 6, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(33, 2, 128, dtype=torch.bfloat16, device="cuda")
    F.flux_qk_norm_rope(ctx, hc, q, None, None, 33, qo, None)
    F.flux_qk_norm_rope(ctx, hc, None, k, None, 33, None, ko)
    near_enough(qo, S.normed(qx, wqx, EPS), S.normed(qx, wqx, EPS), 0, False)
    near_enough(ko, S.normed(kx, wkx, EPS), S.normed(kx, wkx, EPS), 0, False)


@pytest.mark.parametrize("value", [0.0, 2.0 ** 60, 2.0 ** -100, float("inf"), float("nan")])
def test_rows_of_unusual_values(F, ctx, value):
    """What is not finite stays in its row (and, without a norm, in its pair); zeros and small values are not divided by."""
    t, hq, hkv, d, rot = 3, 2, 1, 64, 32
    _, x, _, _ = rows(5, t, hq, hkv, d)
    x[1, 0, 5] = value
    if value < 1:
        x[1, 0] = value
    if value == 2.0 ** 60:
        x[1, 0] *= 2.0 ** 60
    dev, x = bf16(x)
    f, fx = freqs(rot)
    (wq, wk), (wqx, _) = weights(5, d)
    for norm in (True, False):
        out = torch.empty(t, hq, d, dtype=torch.bfloat16, device="cuda")
        F.flux_qk_norm_rope(ctx, F.head_cfg(hq, hkv, d, wq if norm else None, wk if norm else None, EPS, f), dev[:, :hq], None, i32([1, 2, 3]), t, out, None)
        with np.errstate(all="ignore"):
            n = S.normed(x[:, :hq], wqx if norm else None, EPS)
            want = S.turned(n, [1, 2, 3], fx, False)
        fine = np.isfinite(want)
        assert np.array_equal(torch.isfinite(out).cpu().numpy(), fine)
        near_enough(torch.where(torch.from_numpy(fine).cuda(), out, 0), np.where(fine, want, 0), np.where(np.isfinite(n), n, 0), rot, False)


# ---- into the contiguous cache ---------------------------------------------------------------------------------------

def append_case(F, ctx, seed, lens, new, hq, hkv, d, rot, near, norm, cap, positions=None, extra=0, no_q=False, **at):
    t = sum(new)
    dev, _, (q, k, v), (qx, kx, vx) = rows(seed, t + extra, hq, hkv, d)
    (wq, wk), (wqx, wkx) = weights(seed, d, norm)
    f, fx = freqs(rot) if rot else (None, None)
    hc = F.head_cfg(hq, hkv, d, wq, wk, EPS, f, rot, near)
    cache = F.KVCache(*(torch.full((len(lens), hkv, cap, d), -3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)), i32(lens))
    out = torch.full((t + extra, hq, d), -7.0, dtype=torch.bfloat16, device="cuda")
    F.flux_qkv_append(ctx, hc, cache, None if no_q else q, k, v, cu_of(new), t + extra, max(new), None if positions is None else i32(positions), None if no_q else out, **at)
    place = [(b, n + i) for b, (n, m) in enumerate(zip(lens, new)) for i in range(m)]
    pos = [p for _, p in place] if positions is None else positions
    if not no_q:
        n = S.normed(qx[:t], wqx, EPS)
        near_enough(out[:t], n if not rot else S.turned(n, pos, fx, near), n, rot, near)
    assert bool((out[0 if no_q else t:] == -7.0).all())
    n = S.normed(kx[:t], wkx, EPS)
    want = n if not rot else S.turned(n, pos, fx, near)
    kept = [i for i, (b, p) in enumerate(place) if p < cap]
    bs, ps = i32([place[i][0] for i in kept]).long(), i32([place[i][1] for i in kept]).long()
    near_enough(cache.k[bs, :, ps], want[kept], n[kept], rot, near)
    assert torch.equal(cache.v[bs, :, ps], v[kept])
    untouched = torch.ones(len(lens), cap, dtype=torch.bool, device="cuda")
    untouched[bs, ps] = False
    for c in (cache.k, cache.v):
        assert bool((c.transpose(1, 2)[untouched] == -3.0).all())
    assert cache.kv_len.tolist() == [min(cap, a + b) for a, b in zip(lens, new)]
    return len(kept) < t


@pytest.mark.parametrize("lens,new,hq,hkv,d,rot,near,norm", [
    ([0], [1], 8, 2, 64, 64, 0, True),
    ([5, 0, 17], [1, 1, 1], 32, 8, 128, 128, 0, True),
    ([5, 0, 17, 3], [0, 40, 1, 0], 28, 4, 128, 64, 0, False),
    ([3, 100], [700, 301], 6, 3, 64, 32, 1, True),
    ([i % 7 for i in range(64)], [i % 3 for i in range(64)], 4, 1, 64, 64, 0, True),
    ([i % 7 for i in range(65)], [(i + 1) % 3 for i in range(65)], 4, 1, 64, 64, 1, True),
    ([i % 9 for i in range(4200)], [(i * 7) % 3 for i in range(4200)], 1, 1, 64, 16, 0, False),
])
def test_append(F, ctx, lens, new, hq, hkv, d, rot, near, norm):
    assert not append_case(F, ctx, len(lens), lens, new, hq, hkv, d, rot, near, norm, max(a + b for a, b in zip(lens, new)) + 3)
    assert F.flux_last_device_status(ctx) == 0


def test_append_where_the_cache_ends(F, ctx):
    assert append_case(F, ctx, 1, [10, 60, 64], [3, 9, 2], 8, 2, 64, 64, 0, True, 64)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_KV_OVERFLOW


def test_append_with_other_positions_rows_of_no_sequence_and_no_queries(F, ctx):
    append_case(F, ctx, 2, [4, 9], [6, 5], 8, 2, 64, 64, 0, True, 40, positions=[100 * i for i in range(11)])
    append_case(F, ctx, 3, [4, 9], [6, 5], 8, 2, 64, 64, 0, True, 40, extra=7)
    append_case(F, ctx, 4, [4, 9], [6, 50], 8, 2, 64, 0, 0, True, 70, no_q=True)
    assert F.flux_last_device_status(ctx) == 0


def test_append_on_a_strided_cache_and_another_stream(F, ctx):
    """Token-major storage of more heads than the call has; the same as the call in two steps, bit for bit."""
    t, hq, hkv, d = 130, 8, 2, 128
    _, _, (q, k, v), _ = rows(8, t, hq, hkv, d)
    (wq, wk), _ = weights(8, d)
    f, _ = freqs(d)
    hc = F.head_cfg(hq, hkv, d, wq, wk, EPS, f)
    store = torch.zeros(2, 2, 300, 5, d, dtype=torch.bfloat16, device="cuda")            # [k or v, batch, t, heads, d]
    cache = F.KVCache(store[0, :, :, 1:3].transpose(1, 2), store[1, :, :, 1:3].transpose(1, 2), i32([20, 0]))
    other = F.KVCache.empty(2, hkv, 300, d)
    other.k.zero_(), other.v.zero_(), other.kv_len.copy_(i32([20, 0]))
    cu, out, out2 = cu_of([100, 30]), torch.empty(t, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(t, hq, d, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    F.flux_qkv_append(ctx, hc, cache, q, k, v, cu, t, 100, None, out, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    pos = torch.cat([torch.arange(20, 120), torch.arange(30)]).to(torch.int32).cuda()
    k2 = torch.empty(t, hkv, d, dtype=torch.bfloat16, device="cuda")
    F.flux_qk_norm_rope(ctx, hc, q, k, pos, t, out2, k2)
    F.flux_kv_append(ctx, other, hkv, d, k2, v.contiguous(), cu, t, 100)
    assert torch.equal(out, out2) and torch.equal(cache.k, other.k) and torch.equal(cache.v, other.v) and torch.equal(cache.kv_len, other.kv_len)
    assert not store[:, :, :, 0].any() and not store[:, :, :, 3:].any()


# ---- into pages ------------------------------------------------------------------------------------------------------

def pool_of(F, seed, n, hkv, d):
    rng = np.random.default_rng(seed)
    codes = [rng.integers(0, 0x7F, (n, hkv, 64, d)).astype(np.uint8) for _ in range(2)]
    scale = [np.exp2(rng.integers(-9, -6, (n, hkv))).astype(np.float32) for _ in range(2)]
    return F.PagedKV(*(torch.from_numpy(c.copy()).cuda() for c in codes), *(torch.from_numpy(s.copy()).cuda() for s in scale)), codes, scale


@pytest.mark.parametrize("new,first,hq,hkv,d,rot,near,norm,scale", [
    ([1], [0], 8, 2, 64, 64, 0, True, 1.0),
    ([1, 1, 1], [63, 0, 17], 32, 8, 128, 128, 0, True, 1.0),
    ([64, 100, 3], [0, 60, 5], 28, 4, 128, 64, 0, False, 3.0),
    ([200, 1, 129], [7, 63, 0], 6, 3, 64, 32, 1, True, 1.0),
    ([130], [1], 4, 2, 128, 128, 1, False, 1e-12),
    ([70], [3], 4, 2, 64, 0, 0, True, 1.0),
    ([1] * 150, [i % 64 for i in range(150)], 4, 1, 64, 64, 0, True, 1.0),
])
def test_append_paged(F, ctx, new, first, hq, hkv, d, rot, near, norm, scale):
    t = sum(new)
    dev, _, (q, k, v), (qx, kx, vx) = rows(t, t, hq, hkv, d, scale)
    (wq, wk), (wqx, wkx) = weights(t, d, norm)
    f, fx = freqs(rot) if rot else (None, None)
    held = [-(-(a + b) // 64) for a, b in zip(first, new)]
    ids = np.random.default_rng(t).permutation(sum(held) + 2)
    slots, at = [], 0
    for n, r, h in zip(new, first, held):
        slots += [int(ids[at + (r + i) // 64]) * 64 + (r + i) % 64 for i in range(n)]
        at += h
    slots = [-1, -1] + slots[2:] if t > 140 else slots        # (rows without a place)
    pos = np.random.default_rng(t).integers(0, 100000, t)
    kv, codes, scales = pool_of(F, t, sum(held) + 2, hkv, d)
    out = torch.full((t + 1, hq, d), -7.0, dtype=torch.bfloat16, device="cuda")
    F.flux_qkv_append_paged(ctx, F.head_cfg(hq, hkv, d, wq, wk, EPS, f, rot, near), kv, q, k, v, i32(slots), i32(pos) if rot else None, t, out)
    n = S.normed(qx, wqx, EPS)
    near_enough(out[:t], n if not rot else S.turned(n, pos, fx, near), n, rot, near)
    assert bool((out[t] == -7.0).all())
    want = S.heads(kx, wkx, EPS, pos, fx, near)
    for got, got_scale, c, s, y in ((kv.k, kv.k_scale, codes[0], scales[0], want), (kv.v, kv.v_scale, codes[1], scales[1], vx)):
        P.append(c, s, y, slots)
        assert np.array_equal(got_scale.cpu().numpy(), s)
        assert np.array_equal(got.cpu().numpy() & 0x7F, c & 0x7F) and np.array_equal(P.VALUES[got.cpu().numpy()], P.VALUES[c])
    assert F.flux_last_device_status(ctx) == 0


def test_append_paged_without_queries_and_values_as_the_plain_call(F, ctx):
    """Without norm and rotation the pages are those of flux_kv_append_paged, bit for bit, values that are not finite among them."""
    t, hkv, d = 90, 2, 64
    _, x, _, _ = rows(9, t, 1, hkv, d)
    x[3, 1, 7], x[40, 2, 9], x[66, 3, 0], x[70, 4, 1] = np.inf, np.nan, -np.inf, 1e30
    dev, _ = bf16(x)
    k, v = dev[:, 1:3], dev[:, 3:]
    slots = i32(list(range(64 * 3 + 5, 64 * 4)) + list(range(64, 64 + 31)))
    a, _, _ = pool_of(F, 1, 5, hkv, d)
    b, _, _ = pool_of(F, 1, 5, hkv, d)
    F.flux_qkv_append_paged(ctx, F.head_cfg(1, hkv, d), a, None, k, v, slots, None, t, None)
    F.flux_kv_append_paged(ctx, b, hkv, d, k.contiguous(), v.contiguous(), slots, t)
    for p, q in ((a.k, b.k), (a.v, b.v)):
        assert torch.equal(p & 0x7F, q & 0x7F)                # (the sign of NaN is nobody's)
        assert bool(((p == q) | ((p & 0x7F) == 0x7F)).all())
    assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)


def test_append_paged_with_slots_outside_the_pool(F, ctx):
    t, hkv, d = 4, 2, 64
    _, _, (q, k, v), _ = rows(10, t, 1, hkv, d)
    kv, codes, _ = pool_of(F, 2, 3, hkv, d)
    F.flux_qkv_append_paged(ctx, F.head_cfg(1, hkv, d), kv, None, k, v, i32([3 * 64, 3 * 64 + 1, -5, 1 << 30]), None, t, None)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    assert np.array_equal(kv.k.cpu().numpy(), codes[0]) and np.array_equal(kv.v.cpu().numpy(), codes[1])
