"""The cache's bookkeeping (eb_kv_extend): sums of a batch that are large, and steps with fewer
rows than tokens, alone and with the attention after them."""
import numpy as np
import pytest
import torch

from tests import attention_helpers as A
from tests import kv_helpers as K

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


# ---------------------------------------------------------------------------
# fewer rows than tokens
# ---------------------------------------------------------------------------

def _run(eb, c):
    table = A.ints(c["table"])
    b = eb.kv_extend(table, A.ints(c["cached"]), A.ints(c["added"]), A.ints(c["free"]), A.ints([c["n_free"]]),
                     c["page"], c["pages"], c["rows"])
    got = dict(table=table, q_start=b.q_start, kv_len=b.kv_len, slots=b.slots, positions=b.positions,
               n_free=b.n_free, short=b.short)
    want = K.extend_ref(c["table"], c["cached"], c["added"], c["free"], c["n_free"], c["page"], c["pages"], c["rows"])
    torch.cuda.synchronize()
    for name, g in got.items():
        assert np.array_equal(g.cpu().numpy(), np.asarray(want[name])), name


LENS = [(10, 30), (0, 100), (40, 5), (7, 0), (0, 17)]


@pytest.mark.parametrize("rows", [0, 1, 6, 7, 29, 30, 31, 61, 94, 129, 130, 134, 135, 136, 151, 152, 153])
def test_extend_fewer_rows(eb, rows):
    """The last tokens of a batch that has more of them than the step has rows do not join."""
    _run(eb, K.extend_case(LENS, 16, seed=rows, rows=rows))
    _run(eb, K.extend_case(LENS, 16, seed=rows, rows=rows, n_free=4))
    _run(eb, K.extend_case(LENS, 16, seed=rows, rows=rows, stride=3))
    c = K.extend_case(LENS, 16, seed=rows, rows=rows)
    c["free"][-2], c["free"][-4] = -1, c["pages"]
    _run(eb, c)


@pytest.mark.parametrize("batch", [3, 511, 512, 513, 1500, 4096])
@pytest.mark.parametrize("share", [0.02, 0.5, 0.97])
def test_extend_fewer_rows_of_many_sequences(eb, batch, share):
    rng = np.random.default_rng(batch)
    lens = [(int(rng.integers(0, 200)), int(rng.integers(0, 60) if rng.random() < 0.4 else rng.integers(0, 2)))
            for _ in range(batch)]
    _run(eb, K.extend_case(lens, 16, seed=batch, rows=int(share * sum(a for _, a in lens))))


def test_extend_wild_values(eb):
    """What the stack, the table and the lengths may hold beside the ordinary."""
    for n_free in (0, 1, 3, 5, 1 << 30, -5):
        _run(eb, K.extend_case(LENS, 16, seed=n_free & 15, n_free=n_free))
    c = K.extend_case(LENS, 16, seed=9)
    c["free"][-2], c["free"][-4] = -1, c["pages"]
    _run(eb, c)
    c["table"][0, 0] = c["pages"] + 3      # the page that sequence 0 has begun
    _run(eb, c)
    _run(eb, K.extend_case(LENS, 16, seed=10, stride=3))
    _run(eb, K.extend_case([(-4, 20), (8, -3), (3, 2)], 16, seed=12))
    _run(eb, dict(table=np.zeros((2, 4), np.int32), cached=np.array([2 ** 31 - 1, 3]), added=np.array([0, 2]),
                  free=np.array([1, 2], np.int32), n_free=2, page=16, pages=8, rows=4))


def test_steps_of_a_fixed_row_count(eb):
    """A captured step of 24 rows takes prompts as far as its rows go and the rest in the next
    replays: the attention of every token is that of its whole sequence, no page is lost, and
    what stale entries name (pages of another sequence) is neither read nor written."""
    page, pages, rows, hq, hkv, d, total = 16, 40, 24, 4, 2, 64, [50, 9, 37]
    gen = torch.Generator().manual_seed(3)
    x = [torch.randn(t, (hq + 2 * hkv) * d, generator=gen).to(torch.bfloat16).to(DEV) for t in total]
    cache = eb.empty_kv_cache(pages, page, hkv, d)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    other = 39   # the page of a sequence that is not in this batch
    cache.k[other], cache.v[other] = 7.0, 7.0
    order = np.random.default_rng(0).permutation(pages - 1).astype(np.int32)
    free = A.ints(order)
    table = torch.full((3, 4), other, dtype=torch.int32, device=DEV)   # stale entries
    cached, added, n_free = A.ints([0] * 3), A.ints([0] * 3), A.ints([pages - 1])
    qkv = torch.zeros(rows, (hq + 2 * hkv) * d, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(rows, hq, d, dtype=torch.bfloat16, device=DEV)

    def step():
        b = eb.kv_extend(table, cached, added, free, n_free, page, pages, rows)
        q = eb.rope_append(qkv, cache, b.slots, b.positions, None, hq)
        eb.attention(q, cache, table, b.q_start, b.kv_len, rows, 64, out=out)
        return b

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b = step()
    done, outs = [0] * 3, [[], [], []]
    while done != total:
        want = [min(t - n, 30) for t, n in zip(total, done)]     # more than the step has rows
        added.copy_(A.ints(want))
        packed = torch.cat([s[n:n + w] for s, n, w in zip(x, done, want)])[:rows]
        qkv.zero_()
        qkv[:len(packed)] = packed
        graph.replay()
        torch.cuda.synchronize()
        q_start, now = b.q_start.tolist(), b.kv_len.tolist()
        assert [n - m for n, m in zip(now, done)] == [e - s for s, e in zip(q_start, q_start[1:])]
        assert int(b.short) == sum(want) - q_start[-1] and q_start[-1] == min(sum(want), rows)
        for i in range(3):
            outs[i].append(out[q_start[i]:q_start[i + 1]].clone())
        assert int(b.n_free) == pages - 1 - sum(-(-n // page) for n in now)
        cached.copy_(b.kv_len)
        n_free.copy_(b.n_free)
        done = now
    assert bool((cache.k[other] == 7.0).all()) and bool((cache.v[other] == 7.0).all())
    for i, t in enumerate(total):
        q, k, v = x[i].view(t, -1, d).split((hq, hkv, hkv), 1)
        one = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
        keys = [c.transpose(0, 1).reshape(1, hkv, t, d) for c in (k, v)]
        pad = [torch.cat([c, torch.zeros(1, hkv, 64 - t, d, dtype=c.dtype, device=DEV)], 2) for c in keys]
        ref, err = A.attn_ref(q, pad[0].contiguous(), pad[1].contiguous(), one, A.starts([t]), A.ints([t]))
        A.assert_attn(torch.cat(outs[i]), ref, err, f"sequence {i}")
