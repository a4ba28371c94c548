"""Which kernel attention takes (eb_attention_plan), without a GPU: 256 CUs are assumed there."""
import ctypes

import pytest

from tests.test_attention_cpu import GB, _attn_op, eb  # noqa: F401


def _plan(eb, **kw):  # noqa: F811
    rows, splits = ctypes.c_int32(-1), ctypes.c_int32(-1)
    st = eb.lib.eb_attention_plan(ctypes.byref(_attn_op(eb, prefix=0, **kw)), ctypes.byref(rows), ctypes.byref(splits))
    return (rows.value, splits.value) if st == 0 else st


def _heads(hq, hkv):
    return dict(q_heads=hq, cache_heads=hkv, q_stride=hq * 128, out_stride=hq * 128, batch=1)


def test_kernel_by_sizes(eb):  # noqa: F811
    few = dict(_heads(32, 8), rows=1, max_new=1)
    assert _plan(eb, max_kv=64, **few) == (32, 0)
    assert _plan(eb, max_kv=8000, **few)[0] == 32 and _plan(eb, max_kv=8000, **few)[1] > 0
    long = dict(_heads(32, 8), rows=4096, max_new=4096)
    assert _plan(eb, max_kv=4096, **long) == (128, 0)
    chunk = dict(_heads(32, 8), rows=256, max_new=256)
    assert _plan(eb, max_kv=16000, **chunk)[0] == 128 and _plan(eb, max_kv=16000, **chunk)[1] > 0


@pytest.mark.parametrize("kw,status", [(dict(rows=0), -1), (dict(max_new=0), -1), (dict(cache_dim=96), -3),
                                       (dict(q=3 * GB + 2), -2), (dict(mask=2), -1)])
def test_refusals(eb, kw, status):  # noqa: F811
    assert _plan(eb, **kw) == status


def test_null_pointers(eb):  # noqa: F811
    op, n = _attn_op(eb), ctypes.c_int32()
    f = eb.lib.eb_attention_plan
    assert f(None, ctypes.byref(n), ctypes.byref(n)) == -1
    assert f(ctypes.byref(op), None, ctypes.byref(n)) == -1 and f(ctypes.byref(op), ctypes.byref(n), None) == -1
