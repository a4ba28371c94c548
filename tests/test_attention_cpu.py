"""The C entry points of include/eb_attention.h without a GPU: every refusal comes
before anything reaches the HIP runtime, and the binding's structures match."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GB = 1 << 30


@pytest.fixture(scope="module")
def eb():
    if not os.path.exists(os.path.join(ROOT, "paper_2607_02501_amd", "libeb.so")):
        from paper_2607_02501_amd import build

        build.build()
    from paper_2607_02501_amd import eb as _eb

    return _eb


def _cache(eb, **kw):
    c = dict(k=1 * GB, v=2 * GB, type=eb.EB_BF16, heads=2, dim=128, page=16, pages=64, reserved=0)
    c.update(kw)
    return eb.eb_kv_cache(*[c[n] for n, _ in eb.eb_kv_cache._fields_])


def _split(eb, kw):
    """Cache fields of kw, written cache_x, and the others."""
    mine = {k[6:]: v for k, v in kw.items() if k.startswith("cache_")}
    return _cache(eb, **mine), {k: v for k, v in kw.items() if not k.startswith("cache_")}


def _extend(eb, **kw):
    o = dict(cached=1 * GB, added=2 * GB, table=3 * GB, free_pages=4 * GB, n_free=5 * GB, n_free_out=6 * GB,
             q_start=7 * GB, kv_len=8 * GB, slots=9 * GB, positions=10 * GB, short_rows=11 * GB, batch=4,
             rows=8, page=16, pages=64, table_stride=10, free_capacity=64)
    o.update(kw)
    op = eb.eb_kv_extend_op(**o)
    return eb.lib.eb_kv_extend(ctypes.byref(op), None)


def _rope(eb, **kw):
    cache, kw = _split(eb, kw)
    o = dict(qkv=3 * GB, q_out=4 * GB, slots=5 * GB, positions=6 * GB, freqs=7 * GB, q_norm=8 * GB,
             k_norm=9 * GB, qkv_stride=12 * 128, q_stride=8 * 128, pos_stride=5, qkv_type=eb.EB_F32, q_heads=8,
             rows=5, rot=128, style=0, n_axes=1, sections=(ctypes.c_int32 * 3)(64, 0, 0), norm_eps=1e-6)
    o.update(kw)
    op = eb.eb_rope_append_op(cache=cache, **o)
    return eb.lib.eb_rope_append(ctypes.byref(op), None)


def _attn_op(eb, **kw):
    cache, kw = _split(eb, kw)
    o = dict(q=3 * GB, out=4 * GB, table=5 * GB, q_start=6 * GB, kv_len=7 * GB, prefix=8 * GB, q_stride=8 * 128,
             out_stride=8 * 128, rows=5, batch=3, q_heads=8, table_stride=10, max_new=3, max_kv=160, mask=0,
             window=0, scale=0.1, softcap=0.0)
    o.update(kw)
    return eb.eb_attention_op(cache=cache, **o)


def _attn(eb, ws=20 * GB, wsb=1 << 30, **kw):
    return eb.lib.eb_attention(ctypes.byref(_attn_op(eb, **kw)), ws, wsb, None)


BAD_CACHE = [(dict(cache_k=0), -1), (dict(cache_v=0), -1), (dict(cache_k=GB + 8), -2), (dict(cache_v=2 * GB + 2), -2),
             (dict(cache_type=0), -3), (dict(cache_type=9), -1), (dict(cache_heads=0), -1),
             (dict(cache_heads=1025), -1), (dict(cache_dim=96), -3), (dict(cache_dim=0), -3),
             (dict(cache_page=8), -1), (dict(cache_page=24), -1), (dict(cache_page=131072), -1),
             (dict(cache_pages=0), -1), (dict(cache_page=65536, cache_pages=32768), -1),
             (dict(cache_reserved=1), -1)]


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), -1), (dict(batch=4097), -1), (dict(rows=-1), -1), (dict(rows=(1 << 24) + 1), -1),
    (dict(page=12), -1), (dict(page=0), -1), (dict(pages=0), -1), (dict(pages=1 << 27), -1),
    (dict(table_stride=0), -1), (dict(table_stride=1 << 27), -1), (dict(free_capacity=-1), -1), (dict(free_capacity=(1 << 27) + 1), -1),
    (dict(cached=0), -1), (dict(added=0), -1), (dict(table=0), -1), (dict(free_pages=0), -1),
    (dict(n_free=0), -1), (dict(n_free_out=0), -1), (dict(q_start=0), -1), (dict(kv_len=0), -1),
    (dict(slots=0), -1), (dict(positions=0), -1), (dict(short_rows=0), -1), (dict(table=3 * GB + 2), -2),
    (dict(slots=9 * GB + 1), -2), (dict(n_free_out=5 * GB), -1), (dict(kv_len=1 * GB), -1),
    (dict(q_start=8 * GB - 16), -1), (dict(positions=9 * GB + 28), -1), (dict(table=4 * GB), -1)])
def test_extend_refusals(eb, kw, status):
    assert _extend(eb, **kw) == status


@pytest.mark.parametrize("kw,status", BAD_CACHE + [
    (dict(q_heads=0), -1), (dict(q_heads=4097), -1), (dict(rows=-1), -1), (dict(rows=(1 << 24) + 1), -1),
    (dict(qkv_stride=12 * 128 - 8), -1), (dict(q_stride=8 * 128 - 8), -1), (dict(qkv_stride=12 * 128 + 4), -2),
    (dict(q_stride=8 * 128 + 2), -2), (dict(qkv_type=3), -1), (dict(rot=4), -1), (dict(rot=136), -1),
    (dict(rot=-8), -1), (dict(style=2), -1), (dict(n_axes=0), -1), (dict(n_axes=4), -1),
    (dict(sections=(ctypes.c_int32 * 3)(63, 0, 0)), -1),
    (dict(n_axes=2, sections=(ctypes.c_int32 * 3)(65, -1, 0)), -1),
    (dict(norm_eps=-1.0), -1), (dict(norm_eps=float("nan")), -1), (dict(pos_stride=4), -1),
    (dict(qkv=0), -1), (dict(q_out=0), -1), (dict(slots=0), -1), (dict(positions=0), -1), (dict(freqs=0), -1),
    (dict(qkv=3 * GB + 8), -2), (dict(q_out=4 * GB + 2), -2), (dict(q_norm=8 * GB + 4), -2),
    (dict(k_norm=9 * GB + 8), -2), (dict(slots=5 * GB + 2), -2), (dict(q_out=3 * GB + 1024), -1),
    (dict(q_out=1 * GB + 64), -1), (dict(cache_v=1 * GB + 4096), -1), (dict(slots=4 * GB + 16), -1)])
def test_rope_refusals(eb, kw, status):
    assert _rope(eb, **kw) == status


@pytest.mark.parametrize("kw,status", BAD_CACHE + [
    (dict(rows=-1), -1), (dict(batch=0), -1), (dict(batch=4097), -1), (dict(q_heads=0), -1), (dict(q_heads=7), -1),
    (dict(q_heads=4098), -1), (dict(q_stride=1016), -1), (dict(out_stride=1016), -1), (dict(q_stride=1028), -2),
    (dict(out_stride=1026), -2), (dict(table_stride=0), -1), (dict(table_stride=1 << 27), -1),
    (dict(rows=1 << 24, q_heads=256, q_stride=1 << 15, out_stride=1 << 15), -1), (dict(max_new=0), -1),
    (dict(max_kv=0), -1), (dict(window=-1), -1), (dict(mask=2), -1),
    (dict(scale=float("inf")), -1), (dict(scale=-65537.0), -1), (dict(scale=float("nan")), -1),
    (dict(softcap=1025.0), -3), (dict(softcap=0.0009), -3), (dict(softcap=-1.0), -1), (dict(softcap=float("nan")), -1), (dict(q=0), -1),
    (dict(out=0), -1), (dict(table=0), -1), (dict(q_start=0), -1), (dict(kv_len=0), -1),
    (dict(q=3 * GB + 2), -2), (dict(out=4 * GB + 8), -2), (dict(prefix=8 * GB + 1), -2), (dict(out=3 * GB), -1),
    (dict(out=1 * GB + 256), -1), (dict(out=5 * GB), -1), (dict(ws=20 * GB + 64), -2), (dict(ws=0, wsb=16), -1),
    (dict(ws=3 * GB), -1), (dict(ws=2 * GB), -1)])
def test_attention_refusals(eb, kw, status):
    assert _attn(eb, **kw) == status


def test_attention_workspace(eb):
    """Needed where keys are split over workgroups or the batch is large; refused if too small."""
    size = eb.lib.eb_attention_workspace_bytes

    def need(**kw):
        return size(ctypes.byref(_attn_op(eb, **kw)))
    assert need(batch=1, rows=1, max_new=1, max_kv=64) == 0          # one unit of keys: one workgroup a head
    split = need(batch=1, rows=1, max_new=1, max_kv=4000)
    assert split > 0 and split % 256 == 0
    assert need(batch=1, rows=4096, max_new=4096, max_kv=4096, q_heads=32, q_stride=4096, out_stride=4096,
                cache_heads=32) == 0                                 # tiles enough for the GPU
    assert need(batch=65, rows=65, max_new=1, max_kv=64) > 0         # its items' tables
    assert need(batch=64, rows=64, max_new=1, max_kv=64) == 0
    op = dict(batch=1, rows=1, max_new=1, max_kv=4000)
    assert _attn(eb, ws=20 * GB, wsb=split - 256, **op) == -1
    assert _attn(eb, ws=None, wsb=0, **op) == -1


def test_no_rows_is_a_no_op(eb):
    assert _rope(eb, rows=0, qkv=0, q_out=0, slots=0, positions=0, freqs=0) == 0
    assert _attn(eb, ws=None, wsb=0, rows=0, q=0, out=0, table=0, q_start=0, kv_len=0) == 0
    for f in (eb.lib.eb_kv_extend, eb.lib.eb_rope_append):
        assert f(None, None) == -1
    assert eb.lib.eb_attention(None, None, 0, None) == -1
    assert eb.lib.eb_attention_workspace_bytes(None) == 0
    op = _attn_op(eb, max_kv=0)
    assert eb.lib.eb_attention_workspace_bytes(ctypes.byref(op)) == 0


def test_binding_checks_tensors(eb):
    """Types, shapes and devices that the library cannot see are refused by the binding."""
    t = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        eb.KVCache(t, t)            # host memory
    with pytest.raises(ValueError):
        eb.kv_extend(torch.zeros(2, 4, dtype=torch.int32), t, t, t, t, 16, 4, 2)
