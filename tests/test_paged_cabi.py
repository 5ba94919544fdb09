"""Argument checks of the paged-cache entry points on a context without a device: what is refused is refused before any launch,
what is valid gets as far as the missing device."""
import ctypes as C

import pytest

from tests.test_cabi import F, nodev, rc_of  # noqa: F401


def table(F, **kw):
    d = dict(table=4096, kv_len=256, free_pages=8192, n_free=64, batch=2, table_pages=4, n_pages=8)
    d.update(kw)
    return F.FluxPageTable(*(d[k] for k in ("table", "kv_len", "free_pages", "n_free", "batch", "table_pages", "n_pages")))


def pool(F, **kw):
    d = dict(k=4096, v=8192, k_scale=256, v_scale=512, stride_p=2 * 64 * 128, stride_h=64 * 128, stride_t=128, n_pages=8)
    d.update(kw)
    return F.FluxPagedKV(*(d[k] for k in ("k", "v", "k_scale", "v_scale", "stride_p", "stride_h", "stride_t", "n_pages")))


BAD_TABLES = [dict(table=None), dict(kv_len=None), dict(batch=0), dict(table_pages=0), dict(n_pages=0), dict(n_pages=-1), dict(table_pages=(1 << 24) + 1),
              dict(n_pages=(1 << 24) + 1)]
BAD_POOLS = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=4104), dict(v=8200), dict(stride_t=112), dict(stride_t=136),
             dict(stride_h=8), dict(stride_p=-16), dict(stride_h=-16), dict(stride_t=(1 << 20) + 16), dict(n_pages=0), dict(n_pages=(1 << 24) + 1)]


def test_page_planning(F, nodev):
    plan = lambda pt=None, ctx=nodev, cu=256, t=5, slots=512: rc_of(F, F.flux_page_plan, ctx, pt or table(F), cu, t, slots)
    assert plan() == F.FLUX_EHIP and plan(t=0) == F.FLUX_EHIP
    assert plan(ctx=None) == plan(cu=None) == plan(slots=None) == plan(t=-1) == plan(t=(1 << 30) + 1) == F.FLUX_EINVAL
    release = lambda pt=None, ctx=nodev, keep=256: rc_of(F, F.flux_page_release, ctx, pt or table(F), keep)
    assert release() == F.FLUX_EHIP
    assert release(ctx=None) == release(keep=None) == F.FLUX_EINVAL
    for kw in BAD_TABLES + [dict(free_pages=None), dict(n_free=None), dict(batch=4097), dict(batch=4096, table_pages=1 << 20)]:
        assert plan(table(F, **kw)) == release(table(F, **kw)) == F.FLUX_EINVAL, kw
    assert plan(table(F, batch=4096, table_pages=(1 << 19) - 1)) == F.FLUX_EHIP
    assert F._lib.flux_page_plan(nodev, None, 256, 5, 512, None) == F.FLUX_EINVAL
    assert F._lib.flux_page_release(nodev, None, 256, None) == F.FLUX_EINVAL


def test_append(F, nodev):
    call = lambda kv=None, ctx=nodev, h=2, d=128, k=4096, v=8192, s=256, t=7: rc_of(F, F.flux_kv_append_paged, ctx, kv or pool(F), h, d, k, v, s, t)
    assert call() == F.FLUX_EHIP and call(t=0) == F.FLUX_EHIP and call(d=64) == F.FLUX_EHIP
    assert call(ctx=None) == call(k=None) == call(v=None) == call(s=None) == F.FLUX_EINVAL
    assert call(d=96) == call(h=0) == call(t=-1) == call(t=(1 << 30) + 1) == call(k=4104) == call(v=8193) == F.FLUX_EINVAL
    for kw in BAD_POOLS:
        assert call(pool(F, **kw)) == F.FLUX_EINVAL, kw
    assert F._lib.flux_kv_append_paged(nodev, None, 2, 128, 4096, 8192, 256, 7, None) == F.FLUX_EINVAL


@pytest.mark.parametrize("prefill", [False, True])
def test_attention(F, nodev, prefill):
    good = F.attn_cfg(8, 2, 128, 4, 16)

    def call(cfg=good, kv=None, pt=None, ctx=nodev, q=4096, cu=768, mq=8, mk=200, mode=512, out=1024):
        kv, pt = kv or pool(F), pt or table(F)
        if prefill:
            return rc_of(F, F.flux_attn_prefill_paged, ctx, cfg, q, cu, mq, mk, kv, pt, mode, out)
        return rc_of(F, F.flux_attn_decode_paged, ctx, cfg, q, mk, kv, pt, mode, out)
    assert call() == F.FLUX_EHIP and call(mk=256) == F.FLUX_EHIP and call(mq=0, mk=0) == F.FLUX_EHIP
    assert call(mk=257) == F.FLUX_ECAPACITY and call(mk=-1) == F.FLUX_EINVAL
    assert call(pt=table(F, free_pages=None, n_free=None)) == F.FLUX_EHIP        # attention takes no free pages
    assert call(pt=table(F, n_pages=9)) == F.FLUX_EINVAL                         # the table may name pages that the pool lacks
    assert call(kv=pool(F, n_pages=9)) == F.FLUX_EHIP
    assert call(ctx=None) == call(q=None) == call(mode=None) == call(out=None) == call(q=4100) == call(out=1032) == F.FLUX_EINVAL
    for c in (F.attn_cfg(8, 3, 128, 4, 16), F.attn_cfg(8, 2, 96, 4, 16), F.attn_cfg(8, 2, 128, -1, 16), F.attn_cfg(8, 2, 128, 4, 0),
              F.attn_cfg(8, 2, 128, 4, 16, out_dtype=3), F.attn_cfg(8, 2, 128, 4, 16, 0.0, 0, 48), F.attn_cfg(8, 2, 128, 4, 16, -1.0),
              F.attn_cfg(8, 2, 128, 4, 16, float("nan"))):
        assert call(c) == F.FLUX_EINVAL
    for kw in BAD_POOLS:
        assert call(kv=pool(F, **kw)) == F.FLUX_EINVAL, kw
    for kw in BAD_TABLES:
        assert call(pt=table(F, **kw)) == F.FLUX_EINVAL, kw
    # sinks and windows near the largest int must not wrap
    big = (1 << 31) - 1
    for blk in (0, 64, 65536):
        assert call(F.attn_cfg(8, 2, 128, big, big, 0.0, 0, blk)) == F.FLUX_EHIP
    # bounds that 32-bit counts do not hold
    wide = dict(table_pages=1 << 24)
    if prefill:
        assert call(cu=None) == call(mq=201) == call(mq=-1) == F.FLUX_EINVAL
        assert call(F.attn_cfg(8, 2, 128, 4, 16), pt=table(F, **wide), mq=1 << 29, mk=1 << 30) == F.FLUX_EINVAL
        assert call(pt=table(F, batch=1 << 20), mq=200) == F.FLUX_EINVAL
        assert call(pt=table(F, batch=1 << 17), mq=8) == F.FLUX_EHIP
    else:
        assert call(pt=table(F, batch=1 << 10, **wide), mk=1 << 30) == F.FLUX_EINVAL
        assert call(pt=table(F, batch=16, **wide), mk=1 << 30) == F.FLUX_EHIP


def test_the_binding_checks_shapes_and_layouts(F):
    import torch
    kv = F.PagedKV.empty(3, 2, 64, device="cpu")
    assert kv.k.shape == (3, 2, 64, 64) and kv.k.dtype == torch.float8_e4m3fn and C.sizeof(F.FluxPagedKV) == len(kv.packed)
    pt = F.PageTable.empty(2, 3, 5, device="cpu")
    assert len(pt.packed) == C.sizeof(F.FluxPageTable) and pt.n_free.tolist() == [3] and pt.free_pages.tolist() == [2, 1, 0]
    k, v, ks, vs = kv.k, kv.v, kv.k_scale, kv.v_scale
    for bad in ((k[:, :, :32], v[:, :, :32], ks, vs), (k, v.view(torch.uint8).transpose(0, 1).contiguous().transpose(0, 1), ks, vs),
                (k.float(), v.float(), ks, vs), (k, v, ks[:, :1], vs), (k, v, ks, vs.t().contiguous().t()), (k, v, ks.double(), vs)):
        with pytest.raises(AssertionError):
            F.PagedKV(*bad)
    t = (pt.table, pt.kv_len, pt.free_pages, pt.n_free)
    for i, bad in ((0, pt.table.t()), (0, pt.table.long()), (1, pt.kv_len[:1]), (2, pt.free_pages[::2]), (3, pt.free_pages)):
        with pytest.raises(AssertionError):
            F.PageTable(*t[:i], bad, *t[i + 1:])
    with pytest.raises(AttributeError):                      # a handle's tensors stay its own
        pt.table = pt.table.clone()


def test_prefill_refuses_more_tiles_than_it_counts(F, nodev):
    """Tiles times KV heads that pass 31 bits, by one and by far."""
    for hkv, mq in ((128, 1 << 30), (1 << 20, 1 << 30), (2 ** 31 - 1, 1 << 30), (1 << 22, 65), (257, 1 << 20)):
        cfg = F.attn_cfg(hkv, hkv, 64, 4, 16)
        pt = table(F, batch=1, table_pages=1 << 24)
        assert rc_of(F, F.flux_attn_prefill_paged, nodev, cfg, 4096, 768, mq, 1 << 30, pool(F), pt, 512, 1024) == F.FLUX_EINVAL, (hkv, mq)
    cfg = F.attn_cfg(128, 128, 64, 4, 16)
    assert rc_of(F, F.flux_attn_prefill_paged, nodev, cfg, 4096, 768, 1 << 20, 1 << 20, pool(F), table(F, batch=1, table_pages=1 << 24), 512, 1024) == F.FLUX_EHIP
