"""What the binding refuses of the calls that norm and turn heads: tensors that do not hold the rows and heads that the call names, which the library would read or
write past their ends.  On a context without a device, whose calls end with FLUX_EHIP when all arguments are in order."""
import pytest
import torch

from tests.test_cabi import F, nodev  # noqa: F401

HQ, HKV, D, T = 4, 2, 64, 3


def tensors():
    x = torch.zeros(T, HQ + 2 * HKV, D, dtype=torch.bfloat16)
    n = torch.arange(T + 1, dtype=torch.int32)
    return dict(q=x[:, :HQ], k=x[:, HQ:HQ + HKV], v=x[:, HQ + HKV:], q_out=torch.zeros(T, HQ, D, dtype=torch.bfloat16), k_out=torch.zeros(T, HKV, D, dtype=torch.bfloat16),
                cu=n, slots=n[:T])


def call(F, ctx, kind, raw=False, total=T, **kw):
    a = {**tensors(), **kw}
    hc = F.FluxHeadCfg(HQ, HKV, D, 0, 0, 0.0, None, None, None) if raw else F.head_cfg(HQ, HKV, D)
    with pytest.raises(F.FluxError) as e:
        if kind == "rows":
            F.flux_qk_norm_rope(ctx, hc, a["q"], a["k"], None, total, a["q_out"], a["k_out"])
        elif kind == "append":
            cache = F.KVCache(*(torch.zeros(2, HKV, 8, D, dtype=torch.bfloat16) for _ in range(2)), torch.zeros(2, dtype=torch.int32))
            F.flux_qkv_append(ctx, hc, cache, a["q"], a["k"], a["v"], a["cu"], total, total, None, a["q_out"])
        else:
            kv = F.PagedKV(*(torch.zeros(2, HKV, 64, D, dtype=torch.uint8) for _ in range(2)), *(torch.zeros(2, HKV) for _ in range(2)))
            F.flux_qkv_append_paged(ctx, hc, kv, a["q"], a["k"], a["v"], a["slots"], None, total, a["q_out"])
    return e.value.code


@pytest.mark.parametrize("kind", ["rows", "append", "paged"])
@pytest.mark.parametrize("raw", [False, True])
def test_rows_have_the_heads_and_the_tokens_that_a_call_names(F, nodev, kind, raw):
    t = tensors()
    assert call(F, nodev, kind, raw) == call(F, nodev, kind, raw, q=None, q_out=None) == F.FLUX_EHIP
    assert call(F, nodev, kind, raw, total=2) == F.FLUX_EHIP                              # (a part of the rows)
    assert call(F, nodev, kind, raw, q_out=t["q_out"].view(T, HQ * D)) == F.FLUX_EHIP
    assert call(F, nodev, kind, raw, q_out=t["q_out"].data_ptr()) == F.FLUX_EHIP
    wide, narrow = torch.zeros(T, HQ, 2 * D, dtype=torch.bfloat16), torch.zeros(T, 1, D, dtype=torch.bfloat16)
    for name in ("q", "k") + (("v",) if kind != "rows" else ()):
        for bad in (narrow, t[name][:T - 1], wide, wide[:, :t[name].shape[1]], torch.zeros(T, t[name].shape[1] + 1, D, dtype=torch.bfloat16)):
            with pytest.raises(AssertionError):
                call(F, nodev, kind, raw, **{name: bad})
    for name in ("q_out",) + (("k_out",) if kind == "rows" else ()):
        for bad in (narrow, t[name][:T - 1], t[name][:, :, :D // 2]):
            with pytest.raises(AssertionError):
                call(F, nodev, kind, raw, **{name: bad})
