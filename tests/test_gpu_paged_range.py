"""Values of any size that the header of the paged cache promises: up to 2^64 in magnitude where weights are as far above their reference as
they may get, and down to the smallest scale that an append writes."""
import numpy as np
import pytest
import torch

from tests import test_paged_precision as R
from tests.test_gpu_paged import FA, F, attention_case, ctx, cu_of  # noqa: F401
from tests import helpers as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["decode", "run", "tile"])
@pytest.mark.parametrize("step", [1.0, 27.0, 45.0])          # log2 by which the weights grow from page to page
def test_results_scale_with_the_values(F, ctx, form, step):
    """Scores of page p are p * step in units of log2 and some noise, so that weights stay below the guard for many pages, or move the
    reference now and then or with every page.  Times 2^55 (the largest value is 2^64 then, nearly) every result is the same to the
    bit, times 2^-100 to what the smallest products lose."""
    hq, hkv, d, n = 8, 2, 64, 1500
    rows = [{"decode": 1, "run": 4, "tile": 40}[form]]
    kv, pt, q, qf, seqs = attention_case(F, [n], hq, hkv, d, seed=3, rows=rows)
    # the first element of a key is the page's number, in codes of two of them for up to 23 pages; that of a query is the step
    q[..., 0] = 1.0
    page = torch.zeros(kv.k.shape[0], device="cuda")
    page[pt.table[0, :24].long()] = torch.arange(24.0, device="cuda").clamp(max=15)   # (0 to 15 are codes)
    kv.k_scale.fill_(0.25)
    kv.k.view(torch.float8_e4m3fn)[:, :, :, 0] = page[:, None, None].to(torch.float8_e4m3fn)
    cfg = F.attn_cfg(hq, hkv, d, 0, 1, 4 * step * float(np.log(2.0)), 1) if step > 1 else F.attn_cfg(hq, hkv, d, 0, 1, 0.0, 1)
    if step > 1:                                             # nothing but the page's number and a little noise
        q[..., 1:] *= 1 / 64
    kv.v_scale.fill_(1.0)
    codes = kv.v.view(torch.float8_e4m3fn)
    held = pt.table[0, :24].long()
    codes[held] = torch.where(codes[held].float().abs().isfinite(), codes[held].float() * 32, 0.0).clamp(-448, 448).to(torch.float8_e4m3fn)
    mode = torch.ones(1, dtype=torch.uint8, device="cuda")
    outs = []
    for e in (0, 55, -100):
        kv.v_scale.fill_(2.0 ** e)
        out = torch.empty(rows[0], hq, d, dtype=torch.float32, device="cuda")
        if form == "decode":
            F.flux_attn_decode_paged(ctx, cfg, q, n, kv, pt, mode, out)
        else:
            F.flux_attn_prefill_paged(ctx, cfg, q, cu_of(rows), rows[0], n, kv, pt, mode, out)
        outs.append(H.torch_to_f64(out))
    assert np.isfinite(outs[0]).all() and np.abs(outs[0]).max() > 0.1
    assert np.array_equal(outs[1], outs[0] * 2.0 ** 55)
    assert R.rel(outs[2] * 2.0 ** 100, outs[0]) <= R.THREE_TERMS
    assert F.flux_last_device_status(ctx) == 0
