"""A decode step of cross attention whose lengths or bounds do not fit the cache: the same keys count as in any other call."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged import F, bf16, ctx, cu_of, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [201, 205, 333, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("bound", [1, 65, 130, 199, 200])
def test_a_length_above_the_capacity_counts_as_the_capacity(F, ctx, length, bound):
    rng, cap, hq, hkv, d = np.random.default_rng(bound), 200, 8, 2, 64
    q, _ = bf16(rng.normal(size=(2, hq, d)))
    k, _ = bf16(rng.normal(size=(2, hkv, cap, d)))
    v, _ = bf16(rng.normal(size=(2, hkv, cap, d)))
    cfg = F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1)
    got, want = (torch.full((2, hq, d), -7.0, device="cuda") for _ in range(2))
    F.flux_attn_cross(ctx, cfg, q, None, 1, bound, F.KVCache(k, v, i32([length, min(bound, 60)])), got)
    assert F.flux_last_device_status(ctx) == (F.FLUX_DEV_BAD_LENGTH if bound < cap else 0)
    F.flux_attn_cross(ctx, cfg, q, None, 1, bound, F.KVCache(k, v, i32([bound, min(bound, 60)])), want)
    assert F.flux_last_device_status(ctx) == 0
    assert torch.equal(got, want)
