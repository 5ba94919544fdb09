"""The definitions the paged cache is tested against, on their own (no GPU)."""
import numpy as np
import torch

from oracle import paged_oracle as P


def test_code_values_are_those_of_torch():
    mine, theirs = P.VALUES, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mine, theirs, equal_nan=True) and np.isnan(mine).sum() == 2 and np.nanmax(mine) == 448


def test_encoding_is_to_nearest_even():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 8, 4000), P.VALUES[~np.isnan(P.VALUES)],
                        (P.VALUES[:126] + P.VALUES[1:127]) / 2])           # the ties
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(P.encode(x.astype(np.float64)), want)
    assert (P.encode(np.array([np.inf, -np.inf, np.nan])) & 0x7F == 0x7F).all()


def test_the_scale_is_the_smallest_power_of_two_that_fits():
    for amax in (448.0, 448.0001, 224.0, 1.0, 1e-3, 3e38, 0.0, 1e-38):
        s = P.scale_for(amax)
        assert amax <= 448 * s and (s == 2.0 ** -100 or amax > 224 * s)


def test_plan_and_release_are_inverse():
    p = P.Pages([[-1] * 5 for _ in range(3)], [0, 0, 0], list(range(9, -1, -1)), 10, 10)
    s, over = p.plan([70, 0, 64])
    assert not over and p.kv_len == [70, 0, 64] and p.n_free == 7 and s[:2] == [0, 1] and s[64] == 64 and s[70] == 128
    before = ([list(r) for r in p.table], list(p.kv_len), list(p.free), p.n_free)
    p.plan([1, 130, 5])
    p.release([70, 0, 64])
    after = ([list(r) for r in p.table], list(p.kv_len), list(p.free), p.n_free)
    assert before == after
    s, over = p.plan([0, 400, 1])
    assert over and p.kv_len == [70, 320, 65] and s[320:400] == [-1] * 80


def test_growing_scales_round_old_codes_again():
    codes, scale = np.zeros((1, 1, 64, 16), np.uint8), np.ones((1, 1), np.float32)
    a, b = np.full((3, 1, 16), 1.0625), np.full((1, 1, 16), 500.0)
    P.append(codes, scale, a, [0, 1, 2])
    assert scale[0, 0] == 2.0 ** -8 and (P.VALUES[codes[0, 0, :3]] * scale[0, 0] == 1.0).all()     # 272 lies between 256 and 288: to even
    P.append(codes, scale, b, [3])
    assert scale[0, 0] == 2.0 and (P.VALUES[codes[0, 0, :3]] == 0.5).all() and (P.VALUES[codes[0, 0, 3]] == 256).all()
