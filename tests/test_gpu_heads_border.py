"""Keys that go into pages as codes, turned by angles that bring a value so near to the border between two codes that a sine or cosine off by 2^-33 puts it on the
other side."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from oracle import serving_oracle as S
from tests.test_gpu_heads import bf16, i32, pool_of
from tests.test_gpu_paged import F, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
PAIRS = 24


def near_borders(seed):
    """PAIRS of (position, frequency in fp32, a, b) whose a cos t - b sin t, t = position * frequency, lies 1.5e-11 to 4e-11 of |a| + |b| off the border
    between two codes of scale 1.  t is near an odd multiple of pi / 4, where a series about the nearest quarter turn leaves most: x^14 / 14! = 4e-13 of a cosine
    that ends at x^12 (x^12 / 12! = 1.2e-10 of one that ends at x^10), x^13 / 13! = 7e-12 of a sine that ends at x^11.  The turns of position * frequency
    are fewer than 4096, which 64 bits hold to 5e-13 of one."""
    rng, found = np.random.default_rng(seed), []
    pos = np.arange(1, 4096, dtype=np.float64)
    while len(found) < PAIRS:
        a, b = 1 + rng.integers(0, 128) / 128, -1 - rng.integers(0, 128) / 128
        border, size = 1.0625 + 0.125 * rng.integers(0, 8), np.hypot(a, b)
        if border >= size:
            continue
        t = (np.arccos(border / size) * rng.choice([-1, 1]) - np.arctan2(b, a)) % (2 * np.pi)     # a cos t - b sin t = size cos(t + atan2(b, a))
        if abs(t % (np.pi / 2) - np.pi / 4) > 0.06:
            continue
        f = (t / pos).astype(np.float32).astype(np.float64)
        off = np.abs(a * np.cos(pos * f) - b * np.sin(pos * f) - border) / (abs(a) + abs(b))
        hits = np.flatnonzero((off > 1.5e-11) & (off < 4e-11))
        if len(hits):
            found.append((int(pos[hits[0]]), f[hits[0]], a, b))
    return found


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("near", [0, 1])
@pytest.mark.parametrize("one", [False, True])
def test_codes_of_turned_keys_next_to_a_border(F, ctx, seed, near, one):
    """A row per pair, alone in its page or all in one; a plain value of 448 makes the scale 1."""
    d, rot, cases = 64, 2 * PAIRS, near_borders(seed)
    x = np.zeros((PAIRS, 2, d))
    x[:, :, d - 1] = 448.0
    for i, (_, _, a, b) in enumerate(cases):
        p, q = (2 * i, 2 * i + 1) if near else (i, i + PAIRS)
        x[i, 0, p], x[i, 0, q] = a, b
    dev, x = bf16(x)
    freq = np.array([f for _, f, _, _ in cases])
    pos = [p for p, _, _, _ in cases]
    slots = [64 + i if one else 64 * i for i in range(PAIRS)]
    kv, codes, scales = pool_of(F, seed, PAIRS, 1, d)
    hc = F.head_cfg(1, 1, d, inv_freq=torch.from_numpy(freq.astype(np.float32)).cuda(), rotary_dim=rot, interleaved=near)
    F.flux_qkv_append_paged(ctx, hc, kv, None, dev[:, :1], dev[:, 1:], i32(slots), i32(pos), PAIRS, None)
    P.append(codes[0], scales[0], S.turned(x[:, :1], pos, freq, near), slots)
    page, row = np.array(slots) // 64, np.array(slots) % 64
    assert (scales[0][page] == 1.0).all() and np.array_equal(kv.k_scale.cpu().numpy(), scales[0])
    got, want = P.VALUES[kv.k.cpu().numpy()[page, 0, row]], P.VALUES[codes[0][page, 0, row]]
    assert np.array_equal(got, want), np.argwhere(got != want)
    assert F.flux_last_device_status(ctx) == 0
