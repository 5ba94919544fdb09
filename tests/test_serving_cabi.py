"""Argument checks of the head, page-moving and cross-attention entry points on a context without a device."""
import ctypes as C

import pytest
import torch

from tests.test_cabi import F, cache_struct, nodev, rc_of  # noqa: F401
from tests.test_paged_cabi import BAD_POOLS, BAD_TABLES, pool, table


def head(F, **kw):
    d = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, rotary_dim=128, interleaved=0, eps=1e-6, q_norm=4096, k_norm=8192, inv_freq=256)
    d.update(kw)
    return F.FluxHeadCfg(*(d[n] for n, _ in F.FluxHeadCfg._fields_))


def rows(F, **kw):
    d = dict(q=4096, k=8192, v=16384, stride_q=12 * 128, stride_k=12 * 128, stride_v=12 * 128)
    d.update(kw)
    return F.FluxQKVRows(*(d[n] for n, _ in F.FluxQKVRows._fields_))


BAD_HEADS = [dict(n_q_heads=0), dict(n_kv_heads=-1), dict(head_dim=96), dict(rotary_dim=-16), dict(rotary_dim=24), dict(rotary_dim=144), dict(interleaved=2),
             dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0), dict(q_norm=4104), dict(k_norm=8), dict(inv_freq=None), dict(inv_freq=260),
             dict(n_q_heads=(1 << 20) + 1)]
BAD_ROWS = [dict(q=4100), dict(k=8), dict(stride_q=8 * 128 - 8), dict(stride_q=12 * 128 + 4), dict(stride_k=2 * 128 - 8), dict(stride_k=-256), dict(stride_k=260)]


@pytest.mark.parametrize("kind", ["rows", "append", "paged"])
def test_heads(F, nodev, kind):
    def call(hc=None, r=None, ctx=nodev, pos=512, t=5, q_out=1024, k_out=2048, cu=768, mx=3, kc=None, kv=None, slots=640):
        hc, r = C.byref(hc or head(F)), C.byref(r or rows(F))
        if kind == "rows":
            return F._lib.flux_qk_norm_rope(ctx, hc, r, pos, t, q_out, k_out, None)
        if kind == "append":
            return F._lib.flux_qkv_append(ctx, hc, C.byref(kc or cache_struct(F)), r, cu, t, mx, pos, q_out, None)
        return F._lib.flux_qkv_append_paged(ctx, hc, C.byref(kv or pool(F)), r, slots, pos, t, q_out, None)
    assert call() == F.FLUX_EHIP and call(head(F, q_norm=None, k_norm=None, eps=0.0)) == F.FLUX_EHIP
    assert call(head(F, rotary_dim=0, inv_freq=None), pos=None) == F.FLUX_EHIP
    assert call(t=0, mx=0) == F.FLUX_EHIP
    assert call(pos=None) == (F.FLUX_EHIP if kind == "append" else F.FLUX_EINVAL)         # (there they follow from the lengths)
    for kw in BAD_HEADS:
        assert call(head(F, **kw)) == F.FLUX_EINVAL, kw
    for kw in BAD_ROWS + ([dict(k=None), dict(v=None), dict(v=24), dict(stride_v=8), dict(stride_v=257)] if kind != "rows" else []):
        assert call(r=rows(F, **kw)) == F.FLUX_EINVAL, kw
    assert call(ctx=None) == call(t=-1) == call(t=(1 << 30) + 1) == call(q_out=None) == call(r=rows(F, q=None)) == call(q_out=1032) == F.FLUX_EINVAL
    assert call(q_out=4096) == F.FLUX_EINVAL                                             # onto itself, with gaps between the rows
    assert call(q_out=4096, r=rows(F, stride_q=8 * 128)) == F.FLUX_EHIP
    if kind == "rows":
        assert call(r=rows(F, k=None), k_out=None) == call(r=rows(F, q=None), q_out=None) == call(r=rows(F, v=None, stride_v=0)) == F.FLUX_EHIP
        assert call(k_out=None) == call(r=rows(F, k=None)) == call(k_out=2056) == call(k_out=8192) == F.FLUX_EINVAL
        assert call(r=rows(F, k=None, q=None), k_out=None, q_out=None) == F.FLUX_EINVAL
        assert F._lib.flux_qk_norm_rope(nodev, None, C.byref(rows(F)), 512, 5, 1024, 2048, None) == F.FLUX_EINVAL
        assert F._lib.flux_qk_norm_rope(nodev, C.byref(head(F)), None, 512, 5, 1024, 2048, None) == F.FLUX_EINVAL
        return
    assert call(r=rows(F, q=None), q_out=None) == F.FLUX_EHIP
    if kind == "append":
        assert call(cu=None) == call(mx=-1) == call(mx=6) == call(kc=cache_struct(F, k=None)) == call(kc=cache_struct(F, stride_t=64)) == F.FLUX_EINVAL
        assert call(t=100, mx=65) == F.FLUX_ECAPACITY
    else:
        assert call(slots=None) == call(t=(1 << 27) + 1) == F.FLUX_EINVAL and call(t=1 << 27) == F.FLUX_EHIP
        for kw in BAD_POOLS:
            assert call(kv=pool(F, **kw)) == F.FLUX_EINVAL, kw


def test_pages(F, nodev):
    fork = lambda pt=None, ctx=nodev, s=256, p=512, k=640, c=768, n=896: rc_of(F, F.flux_page_fork, ctx, pt or table(F), s, p, k, c, n)
    compact = lambda pt=None, ctx=nodev, s=256, m=768, n=896, most=4: rc_of(F, F.flux_page_compact, ctx, pt or table(F), s, m, n, most)
    copy = lambda kv=None, ctx=nodev, h=2, d=128, c=768, n=896, most=4: rc_of(F, F.flux_page_copy, ctx, kv or pool(F), h, d, c, n, most)
    assert fork() == fork(p=None) == fork(k=None) == compact() == compact(s=None) == copy() == copy(n=None) == copy(most=0) == copy(d=64) == F.FLUX_EHIP
    assert fork(ctx=None) == fork(s=None) == fork(c=None) == fork(n=None) == F.FLUX_EINVAL
    assert compact(ctx=None) == compact(m=None) == compact(n=None) == compact(most=0) == compact(most=(1 << 24) + 1) == F.FLUX_EINVAL
    assert copy(ctx=None) == copy(c=None) == copy(h=0) == copy(d=96) == copy(most=-1) == copy(most=(1 << 24) + 1) == F.FLUX_EINVAL
    for kw in BAD_TABLES + [dict(free_pages=None), dict(n_free=None), dict(batch=4097), dict(batch=4096, table_pages=1 << 20)]:
        assert fork(table(F, **kw)) == compact(table(F, **kw)) == F.FLUX_EINVAL, kw
    assert compact(table(F, n_pages=(1 << 20) + 1)) == F.FLUX_EINVAL and compact(table(F, n_pages=1 << 20)) == fork(table(F, n_pages=1 << 24)) == F.FLUX_EHIP
    for kw in BAD_POOLS:
        assert copy(pool(F, **kw)) == F.FLUX_EINVAL, kw


def test_cross(F, nodev):
    good = F.attn_cfg(8, 2, 128, 0, 1)
    call = lambda cfg=good, kc=None, ctx=nodev, q=4096, cu=768, mq=8, mk=32, out=1024: rc_of(F, F.flux_attn_cross, ctx, cfg, q, cu, mq, mk, kc or cache_struct(F), out)
    assert call() == call(cu=None) == call(cu=None, mq=1) == call(mq=500) == call(mk=0) == call(mq=0) == call(mk=64) == F.FLUX_EHIP
    assert call(mk=65) == F.FLUX_ECAPACITY
    assert call(ctx=None) == call(q=None) == call(out=None) == call(q=4104) == call(out=8) == call(mq=-1) == call(mk=-1) == F.FLUX_EINVAL
    for c in (F.attn_cfg(8, 3, 128, 0, 1), F.attn_cfg(8, 2, 96, 0, 1), F.attn_cfg(8, 2, 128, 0, 1, out_dtype=2), F.attn_cfg(8, 2, 128, 0, 1, float("inf"))):
        assert call(c) == F.FLUX_EINVAL
    for kw in (dict(k=None), dict(v=8), dict(kv_len=None), dict(batch=0), dict(capacity=0), dict(stride_t=64), dict(stride_t=(1 << 22) + 8), dict(stride_h=4)):
        assert call(kc=cache_struct(F, **kw)) == F.FLUX_EINVAL, kw
    assert call(mq=1 << 30) == call(cu=None, mq=1 << 20, kc=cache_struct(F, batch=1 << 12)) == F.FLUX_EINVAL


def test_the_binding_checks_shapes(F):
    w, f = torch.ones(64, dtype=torch.bfloat16), torch.ones(16)
    hc = F.head_cfg(4, 2, 64, w, None, 1e-5, f)
    assert hc.rotary_dim == 32 and len(hc.packed) == C.sizeof(F.FluxHeadCfg) and F.head_cfg(4, 2, 64).rotary_dim == 0
    for kw in (dict(q_norm=w.float()), dict(k_norm=w[:32]), dict(inv_freq=f.double()), dict(inv_freq=f, rotary_dim=64), dict(q_norm=torch.ones(128, dtype=torch.bfloat16)[::2])):
        with pytest.raises(AssertionError):
            F.head_cfg(4, 2, 64, **kw)
    x = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    assert len(F._rows_arg(x[:, :4], x[:, 4:6], x[:, 6:])) == C.sizeof(F.FluxQKVRows)
    for bad in (x.float(), x.transpose(0, 1), x[:, ::2], x[..., ::2]):
        with pytest.raises(AssertionError):
            F._rows_arg(bad, None, None)
