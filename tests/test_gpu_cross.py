"""Cross attention on the GPU against its definition in float64."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from tests.test_gpu_paged import F, bf16, ctx, cu_of, i32  # noqa: F401

pytestmark = pytest.mark.gpu


def case(F, ctx, seed, new, keys, hq, hkv, d, fp32=0, even=False, cap=None, scale=0.0, gain=1.0, max_q=None, max_k=None, strided=False, extra=0, stream=None):
    rng = np.random.default_rng(seed)
    t, cap = sum(new), cap or max(max(keys), 1)
    q, qx = bf16(rng.normal(size=(t + extra, hq, d)) * gain)
    k, kx = bf16(rng.normal(size=(len(keys), hkv, cap, d)))
    v, vx = bf16(rng.normal(size=(len(keys), hkv, cap, d)))
    for b, n in enumerate(keys):                             # what lies behind the length is never used
        k[b, :, n:], v[b, :, n:] = float("nan"), float("inf")
    if strided:
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    cfg = F.attn_cfg(hq, hkv, d, 0, 1, scale, fp32)
    out = torch.full((t + extra, hq, d), -7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    F.flux_attn_cross(ctx, cfg, q, None if even else cu_of(new), max(new) if max_q is None else max_q, max(keys) if max_k is None else max_k,
                      F.KVCache(k, v, i32(keys)), out, stream=stream)
    torch.cuda.synchronize()
    got, at = out.double().cpu().numpy(), 0
    assert (got[t:] == -7.0).all()
    worst = 0.0
    for b, (n, m) in enumerate(zip(new, keys)):
        ref, mag = S.cross(qx[at:at + n], kx[b, :, :m].transpose(1, 0, 2), vx[b, :, :m].transpose(1, 0, 2), scale or 1 / np.sqrt(d))
        # Weights are rounded by 2^-8 of one at most, in the sum of values and in their own: twice that of the mean magnitude of the values.  The
        # result is rounded by 2^-8 of it (fp32: nothing to speak of).  Scores, sums and exponentials in fp32: a score of magnitude up to
        # 40 * gain is off by D * 2^-24 of what it is made of, 2^-10 of a weight at most at gain 4.
        tol = (2 * 2.0 ** -8 + 2.0 ** -10) * mag + (0 if fp32 else 2.0 ** -8) * np.abs(ref) + 1e-30
        off = np.abs(got[at:at + n] - ref)
        assert np.isfinite(got[at:at + n]).all() and (off <= tol).all(), (b, n, m, float((off / tol).max()))
        if m == 0:
            assert not got[at:at + n].any()
        elif n:
            worst = max(worst, float(np.sqrt((off ** 2).sum() / (ref ** 2).sum())))
        at += n
    return worst


@pytest.mark.parametrize("new,keys,hq,hkv,d", [
    ([1], [1], 1, 1, 64),
    ([1], [300], 8, 2, 64),
    ([3, 0, 1], [64, 5, 65], 8, 8, 64),
    ([5], [1500], 8, 8, 64),
    ([17, 40, 2], [0, 63, 128], 4, 2, 128),
    ([65], [129], 28, 4, 128),
    ([130, 7], [200, 1000], 12, 1, 128),
    ([129, 1, 64], [31, 700, 0], 32, 8, 128),
    ([700], [40], 32, 8, 64),
    ([300, 20, 5], [2500, 77, 640], 8, 2, 64),
    ([4] * 70, [1 + (37 * i) % 200 for i in range(70)], 4, 2, 64),
    ([i % 3 for i in range(130)], [(53 * i) % 150 for i in range(130)], 8, 4, 128),
    ([2], [20000], 16, 1, 128),
    ([3], [9000], 20, 20, 64),
])
@pytest.mark.parametrize("fp32", [0, 1])
def test_cross(F, ctx, new, keys, hq, hkv, d, fp32):
    case(F, ctx, len(new), new, keys, hq, hkv, d, fp32)
    assert F.flux_last_device_status(ctx) == 0


@pytest.mark.parametrize("n", [1, 2, 5, 33])
@pytest.mark.parametrize("keys", [[1], [100, 0, 7], [1500] * 16, [10 + 3 * i for i in range(66)]])
def test_the_same_rows_for_all(F, ctx, n, keys):
    """No prefix sums; one row each is worked on like a decode step."""
    for hq, hkv, d in ((8, 8, 64), (8, 2, 128)):
        case(F, ctx, n, [n] * len(keys), keys, hq, hkv, d, 0, True)
        case(F, ctx, n, [n] * len(keys), keys, hq, hkv, d, 1, True, cap=1600)
    assert F.flux_last_device_status(ctx) == 0


def test_bounds_strides_and_rows_of_nobody(F, ctx):
    case(F, ctx, 1, [40, 3], [300, 90], 8, 2, 64, cap=500, max_q=400, max_k=500, strided=True, extra=9)
    case(F, ctx, 2, [40, 3], [300, 90], 8, 2, 128, 1, cap=500, max_q=41, max_k=301, strided=True, extra=1)
    case(F, ctx, 3, [200], [333], 8, 2, 128, scale=0.3, gain=1.0)
    case(F, ctx, 4, [2], [5000], 4, 4, 128, 1, scale=0.5, gain=4.0)                       # one key has nearly all of the weight
    assert F.flux_last_device_status(ctx) == 0


def test_rows_and_keys_beyond_the_bounds_are_left_out(F, ctx):
    """As if the sequence were as long as the bound."""
    q, _ = bf16(np.random.default_rng(1).normal(size=(100, 4, 64)))
    k, _ = bf16(np.random.default_rng(2).normal(size=(1, 2, 200, 64)))
    v, _ = bf16(np.random.default_rng(3).normal(size=(1, 2, 200, 64)))
    cfg = F.attn_cfg(4, 2, 64, 0, 1)
    got, want = (torch.full((100, 4, 64), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    F.flux_attn_cross(ctx, cfg, q, cu_of([100]), 70, 130, F.KVCache(k, v, i32([200])), got)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    F.flux_attn_cross(ctx, cfg, q, cu_of([70]), 70, 130, F.KVCache(k, v, i32([130])), want)
    assert torch.equal(got, want) and bool((got[70:] == -7.0).all())
    for n in (-3, 1 << 30):
        F.flux_attn_cross(ctx, cfg, q, cu_of([100]), 100, 200, F.KVCache(k, v, i32([n])), got)
        assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    F.flux_attn_cross(ctx, cfg, q, i32([60, 20]), 100, 200, F.KVCache(k, v, i32([200])), got)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH


def test_a_small_workspace_gives_the_same(F):
    """Whether keys are shared out moves a result by its rounding at most."""
    for bytes_ in (1, 20 << 20):
        c = F.flux_create(0, bytes_)
        case(F, c, 7, [3, 2], [7000, 100], 8, 2, 64)
        case(F, c, 8, [300], [2000], 8, 8, 128)
        torch.cuda.synchronize()
        F.flux_destroy(c)


def test_error_is_that_of_the_roundings(F, ctx):
    """2-norm against float64: a bf16 result and bf16 weights are off by about 1.7e-3 each."""
    assert case(F, ctx, 11, [64], [4000], 8, 2, 128) < 3e-3
    assert case(F, ctx, 12, [1] * 4, [4000] * 4, 8, 2, 128, even=True) < 3e-3


def test_captured_calls_are_replayed(F, ctx):
    """Shared tiles and a decode step in one graph, with other lengths at every replay and eager calls between."""
    rng = np.random.default_rng(5)
    b, n, hq, hkv, d, cap = 3, 4, 8, 2, 64, 3000
    q, _ = bf16(rng.normal(size=(b * n, hq, d)))
    k, _ = bf16(rng.normal(size=(b, hkv, cap, d)))
    v, _ = bf16(rng.normal(size=(b, hkv, cap, d)))
    cfg, lens = F.attn_cfg(hq, hkv, d, 0, 1), i32([1] * b)
    cache = F.KVCache(k, v, lens)

    def calls(x, y):
        F.flux_attn_cross(ctx, cfg, q, None, n, cap, cache, x)
        F.flux_attn_cross(ctx, cfg, q, None, 1, cap, cache, y)
    outs = [torch.empty(b * n, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    want = [torch.empty_like(x) for x in outs]
    calls(*outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(*outs)
    for sizes in ([3000, 10, 0], [1, 2999, 64], [700, 700, 700], [0, 0, 5]):
        lens.copy_(i32(sizes))
        graph.replay()
        calls(*want)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1][:b], want[1][:b])
    assert F.flux_last_device_status(ctx) == 0


def test_on_another_stream_and_beside_prefill(F, ctx):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        case(F, ctx, 21, [33, 2], [400, 1000], 8, 2, 64)
    # queries at the end of a cache of equal length see the same keys as a decode step does
    q, _ = bf16(np.random.default_rng(1).normal(size=(2, 8, 64)))
    k, _ = bf16(np.random.default_rng(2).normal(size=(2, 2, 500, 64)))
    v, _ = bf16(np.random.default_rng(3).normal(size=(2, 2, 500, 64)))
    cache, cfg = F.KVCache(k, v, i32([500, 77])), F.attn_cfg(8, 2, 64, 0, 1)
    a, b, c = (torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    F.flux_attn_cross(ctx, cfg, q, None, 1, 500, cache, a)
    F.flux_attn_decode(ctx, cfg, q, 500, cache, torch.ones(2, dtype=torch.uint8, device="cuda"), b)
    F.flux_attn_cross(ctx, cfg, q, cu_of([1, 1]), 1, 500, cache, c)
    assert torch.equal(a, b)
    assert (a.float() - c.float()).norm() <= 2.0 ** -7 * a.float().norm()
