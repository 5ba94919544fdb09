"""flux_attn_prefill_paged says when a length passes max_kv_len, whatever form works on its rows."""
import pytest
import torch

from tests.test_gpu_paged import FA, SA, F, attention_case, ctx, cu_of, tolerance  # noqa: F401
from tests.test_gpu_paged_prefill import check, prefill_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2, 60])                       # a run, worked on like a decode call; tiles
@pytest.mark.parametrize("long,bound,mode", [
    (640, 600, FA),                                          # the bound ends in the sequence's last page
    (640, 600, SA),
    (5000, 600, SA),                                         # fewer pages than the bound allows hold all that its queries see
    (5000, 600, FA),
    (600, 600, FA),                                          # as long as the bound: nothing to say
    (600, 600, SA),
])
def test_a_length_above_the_bound_is_reported(F, ctx, n, long, bound, mode):
    hq, hkv, d, lens = 8, 2, 64, [long, 577]
    kv, pt, q, qf, seqs = attention_case(F, lens, hq, hkv, d, seed=long, rows=[n, n])
    out = torch.full((2 * n, hq, d), 7.0, dtype=torch.float32, device="cuda")
    cfg = F.attn_cfg(hq, hkv, d, 16, 100, 0.0, 1)
    F.flux_attn_prefill_paged(ctx, cfg, q, cu_of([n, n]), n, bound, kv, pt, torch.full((2,), mode, dtype=torch.uint8, device="cuda"), out)
    assert F.flux_last_device_status(ctx) == (F.FLUX_DEV_BAD_LENGTH if long > bound else 0)
    ref = prefill_ref(qf, seqs, [n, n], [mode] * 2, 16, 100)
    check(out[n:], ref[n:], tolerance(qf, seqs, d), seqs)    # the other sequence is as it would be
    assert torch.isfinite(out).all()
    if long == bound:
        check(out[:n], ref[:n], tolerance(qf, seqs, d), seqs)
