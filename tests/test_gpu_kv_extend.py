"""The cache's bookkeeping (eb_kv_extend) where the sums of a batch are large."""
import numpy as np
import pytest
import torch

from tests import attention_helpers as A

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def eb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02501_amd import eb as _eb

    return _eb


@pytest.mark.parametrize("batch", [1, 64, 127, 128, 192, 256, 513, 4096])
def test_extend_sums_past_31_bits(eb, batch):
    """Every sequence asks for 2^31 - 1 tokens of a step of 2^24 rows: the sums of the batch
    stop short of 32 bits and the first sequence has all rows."""
    page, pages, stride, rows = 16, 8, 4, 1 << 24
    order = np.random.default_rng(batch).permutation(pages)
    table = torch.full((batch, stride), -7, dtype=torch.int32, device=DEV)
    b = eb.kv_extend(table, A.ints([0] * batch), A.ints([2 ** 31 - 1] * batch), A.ints(order), A.ints([pages]),
                     page, pages, rows)
    assert b.q_start.tolist() == [0] + [rows] * batch
    assert int(b.kv_len[0]) == stride * page
    got = order[::-1][:stride]              # the top of the stack
    assert table[0].tolist() == got.tolist()
    assert bool((table[1:] == -7).all())
    want = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    place = np.arange(stride * page)
    want[:stride * page] = A.ints(got[place // page] * page + place % page)
    assert torch.equal(b.slots, want)
    assert torch.equal(b.positions, torch.arange(rows, dtype=torch.int32, device=DEV))
    assert int(b.short) == 2 ** 31 - 1 if batch > 1 else int(b.short) == 2 ** 31 - 1 - stride * page
