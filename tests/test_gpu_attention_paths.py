"""Attention over the paged cache at the numerical edges of its two kernels, on the GPU,
against the 64-bit reference of tests/attention_helpers.py."""
import numpy as np
import pytest
import torch

from tests import attention_helpers as A

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def eb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02501_amd import eb as _eb

    return _eb


def _randn(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


# ---------------------------------------------------------------------------
# weights far below a row's largest
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("gap", [9, 12, 14, 15, 16, 17.5, 18, 20])
@pytest.mark.parametrize("new,kv,hq,hkv,d,cap", [
    (1, 131071, 2, 1, 64, 0.0), (1, 3000, 8, 2, 128, 0.0), (33, 1200, 4, 4, 256, 0.0), (130, 400, 64, 4, 128, 0.0),
    (40, 700, 256, 4, 64, 40.0), (200, 260, 128, 2, 256, 0.0)])
def test_attn_one_key_far_above_the_others(eb, dtype, gap, new, kv, hq, hkv, d, cap):
    """A key whose value is 0 has nearly all the weight: the output comes from the others, each
    e^-gap of it.  A weight that binary16 cannot hold as a normal number after its exponent is
    raised by 11 is off by half of its smallest step, 2^-25 2^-11 of the largest weight."""
    k, v, table = A.paged([kv], 64, hkv, d, dtype, seed=kv)
    k.zero_()
    v.mul_(0.25).add_(1.0)
    first = int(table[0, 0])
    k[first, :, 0, 0] = 1.0     # place 0, which every token sees
    v[first, :, 0] = 0.0
    q = torch.zeros(new, hq, d, dtype=dtype, device=DEV)
    q[:, :, 0] = float(gap)
    q_start, kv_len = A.starts([new]), A.ints([kv])
    got = eb.attention(q, eb.KVCache(k, v), table, q_start, kv_len, new, kv, softcap=cap, scale=1.0)
    # (query heads of one key/value head are alike here: one of each is compared in full)
    assert torch.equal(got.view(new, hkv, -1, d), got.view(new, hkv, -1, d)[:, :, :1].expand(-1, -1, hq // hkv, -1))
    got, q = got[:, ::hq // hkv], q[:, ::hq // hkv].contiguous()
    ref, err = A.attn_ref(q, k, v, table, q_start, kv_len, softcap=cap, scale=1.0)
    if dtype == FP:
        size = float(v.float().abs().max()) * kv
        err = err + 2.0 ** -36 * size
    A.assert_attn(got, ref, err, f"gap {gap}")


@pytest.mark.parametrize("scale", [0.0, -0.0])
@pytest.mark.parametrize("new,kv,hq,hkv,cap", [(1, 300, 4, 2, 0.0), (130, 400, 64, 4, 0.0), (20, 900, 4, 2, 9.0)])
def test_attn_scale_of_zero(eb, scale, new, kv, hq, hkv, cap):
    """Every key that is seen has the same weight, however large its score would be."""
    k, v, table = A.paged([kv], 16, hkv, 64, BF, seed=kv)
    k.mul_(2.0 ** 50)
    q = _randn(new, hq, 64, seed=2, dtype=BF) * 2.0 ** 50
    q_start, kv_len = A.starts([new]), A.ints([kv])
    got = eb.attention(q, eb.KVCache(k, v), table, q_start, kv_len, new, kv, softcap=cap, scale=scale)
    ref, err = A.attn_ref(q, k, v, table, q_start, kv_len, softcap=cap, scale=scale)
    A.assert_attn(got, ref, err, f"scale {scale}")
