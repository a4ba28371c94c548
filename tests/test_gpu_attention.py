"""Attention over the paged cache, head rotation with the cache write, and the
cache's bookkeeping, on the GPU, against the 64-bit references of
tests/attention_helpers.py; and the three together between QKV and O projections."""
import numpy as np
import pytest
import torch

from paper_2607_02501_amd import workloads as W
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
# kv_extend
# ---------------------------------------------------------------------------

def _extend_case(lens, page, seed, spare=2, stride=None, extra_rows=0, n_free=None):
    """lens: (cached, added); pages in shuffled order."""
    rng = np.random.default_rng(seed)
    held = [-(-max(c, 0) // page) for c, _ in lens]
    need = sum(-(-(max(c, 0) + max(a, 0)) // page) for c, a in lens) - sum(held)
    pages = sum(held) + max(need, 0) + spare
    order = rng.permutation(pages).astype(np.int32)
    stride = stride or max(1, max(-(-(max(c, 0) + max(a, 0)) // page) for c, a in lens))
    table, at = np.full((len(lens), stride), -7, np.int32), 0
    for b, h in enumerate(held):
        table[b, :min(h, stride)] = order[at:at + h][:stride]
        at += h
    free = order[at:]
    rows = sum(max(a, 0) for _, a in lens) + extra_rows
    return dict(table=table, cached=np.array([c for c, _ in lens]), added=np.array([a for _, a in lens]),
                free=free, n_free=len(free) if n_free is None else n_free, page=page, pages=pages, rows=rows)


def _run_extend(eb, c):
    table = A.ints(c["table"])
    b = eb.kv_extend(table, A.ints(c["cached"]), A.ints(c["added"]), A.ints(c["free"]),
                     A.ints([c["n_free"]]), page=c["page"], pages=c["pages"], rows=c["rows"])
    got = dict(table=table, q_start=b.q_start, kv_len=b.kv_len, slots=b.slots, positions=b.positions,
               n_free=b.n_free, short=b.short)
    want = A.extend_ref(c["table"], c["cached"], c["added"], c["free"], c["n_free"], c["page"],
                        c["pages"], c["rows"])
    torch.cuda.synchronize()
    for name, g in got.items():
        assert np.array_equal(g.cpu().numpy(), np.asarray(want[name])), name


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("lens", [
    [(0, 1)], [(5, 1)], [(15, 1), (16, 1), (17, 1)], [(0, 0)], [(0, 0), (3, 0), (0, 7), (2, 0)],
    [(0, 100), (31, 33), (1, 0), (64, 64)], [(1000, 1), (0, 513), (16, 16)]])
def test_extend_small(eb, page, lens):
    _run_extend(eb, _extend_case(lens, page, seed=len(lens)))


@pytest.mark.parametrize("batch", [255, 256, 257, 1000, 4096])
def test_extend_many_sequences(eb, batch):
    rng = np.random.default_rng(batch)
    lens = [(int(rng.integers(0, 200)), int(rng.integers(0, 30) if rng.random() < 0.3 else rng.integers(0, 2)))
            for _ in range(batch)]
    _run_extend(eb, _extend_case(lens, 16, seed=batch, extra_rows=77))


def test_extend_runs_out(eb):
    """No pages left, entries that are no pages, table rows that end, fewer rows than tokens,
    negative lengths: slots of -1, and the tokens without a page counted."""
    lens = [(10, 30), (0, 100), (40, 5), (7, 0), (0, 17)]
    for n_free in (0, 1, 3, 5):
        _run_extend(eb, _extend_case(lens, 16, seed=n_free, n_free=n_free))
    c = _extend_case(lens, 16, seed=9)
    c["free"][-2], c["free"][-4] = -1, c["pages"]
    _run_extend(eb, c)
    c["table"][0, 0] = c["pages"] + 3      # the page that sequence 0 has begun
    _run_extend(eb, c)
    _run_extend(eb, _extend_case(lens, 16, seed=10, stride=3))
    c = _extend_case(lens, 16, seed=11)
    c["rows"] = 61
    _run_extend(eb, c)
    c["rows"] = 0
    _run_extend(eb, c)
    _run_extend(eb, _extend_case([(-4, 20), (8, -3), (3, 2)], 16, seed=12))
    c = _extend_case(lens, 16, seed=13, n_free=1 << 30)   # clamped to the stack
    _run_extend(eb, c)
    c = _extend_case(lens, 16, seed=14, n_free=-5)
    _run_extend(eb, c)
    # lengths near the end of 31 bits
    c = dict(table=np.zeros((2, 4), np.int32), cached=np.array([2 ** 31 - 1, 3]), added=np.array([0, 2]),
             free=np.array([1, 2], np.int32), n_free=2, page=16, pages=8, rows=4)
    _run_extend(eb, c)


# ---------------------------------------------------------------------------
# rope_append
# ---------------------------------------------------------------------------

def _rope(eb, rows, hq, hkv, d, xdt, cdt, norm, style, rot, sections, page=16, seed=1, pos=None, pad=0,
          wide=0):
    x = (_randn(rows, (hq + 2 * hkv) * d + wide, seed=seed) * 1.5).to(xdt)
    x = x[:, :(hq + 2 * hkv) * d]
    half = rot // 2
    freqs = (1e4 ** (-torch.arange(half) / max(half, 1))).float().to(DEV) if half else None
    if pos is None:
        pos = torch.randint(0, 40000, (len(sections), rows), dtype=torch.int32,
                            generator=torch.Generator().manual_seed(seed)).to(DEV)
    pages = -(-rows // page) + 2
    cache = eb.KVCache(torch.full((pages, hkv, page, d), 7.0, dtype=cdt, device=DEV),
                       torch.full((pages, hkv, page, d), 7.0, dtype=cdt, device=DEV))
    slots = np.random.default_rng(seed).permutation(pages * page)[:rows].astype(np.int32)
    if pad:
        slots[rows - pad:] = [-1, pages * page, -2 ** 31, 2 ** 31 - 1][:pad]
    gq = 1 + 0.1 * _randn(d, seed=seed + 1) if norm in ("both", "q") else None
    gk = 1 + 0.1 * _randn(d, seed=seed + 2) if norm in ("both", "k") else None
    out = torch.full((rows, hq, d), 7.0, dtype=cdt, device=DEV)
    got = eb.rope_append(x, cache, A.ints(slots), pos if half else None, freqs, hq, gq, gk, 1e-6, style,
                         sections if half else None, out=out)
    torch.cuda.synchronize()
    q, k, v, sq, sk = A.rope_ref(x, hq, hkv, d, pos, freqs, style, sections, gq, gk, 1e-6)
    live = rows - pad
    A.assert_rope(got[:live], q[:live], sq[:live], "q")
    assert bool((got[live:] == 7.0).all())
    s = torch.from_numpy(slots[:live]).long()
    kc, vc = cache.k.cpu(), cache.v.cpu()
    A.assert_rope(kc[s // page, :, s % page], k[:live], sk[:live], "k")
    A.assert_rope(vc[s // page, :, s % page], v[:live], 0 * v[:live], "v")
    other = torch.ones(pages * page, dtype=torch.bool)
    other[s] = False
    for c in (kc, vc):
        assert bool((c.transpose(1, 2).reshape(pages * page, -1)[other] == 7.0).all())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("style", ["half", "adjacent"])
@pytest.mark.parametrize("xdt,cdt", [(torch.float32, BF), (torch.float32, FP), (BF, BF), (FP, FP), (BF, FP), (FP, BF)])
def test_rope_types(eb, d, style, xdt, cdt):
    _rope(eb, 5, 6, 2, d, xdt, cdt, "both", style, d, (d // 2,), seed=d)


@pytest.mark.parametrize("rows,hq,hkv,d,rot,sections,norm,pad,wide", [
    (1, 1, 1, 64, 64, (32,), None, 0, 0), (1, 32, 32, 128, 128, (64,), None, 0, 0),
    (3, 7, 1, 64, 40, (5, 8, 7), "q", 0, 8), (9, 5, 3, 128, 8, (4,), "k", 4, 0),
    (17, 8, 1, 256, 232, (50, 66), "both", 2, 64), (2, 24, 24, 128, 128, (16, 24, 24), "both", 0, 0),
    (50, 3, 3, 64, 0, (0,), "both", 1, 0), (300, 9, 1, 128, 96, (0, 48, 0), None, 3, 16),
    (2049, 2, 1, 64, 64, (32,), "both", 0, 0), (130, 40, 8, 128, 128, (22, 42), None, 0, 0)])
@pytest.mark.parametrize("style", ["half", "adjacent"])
def test_rope_layouts(eb, rows, hq, hkv, d, rot, sections, norm, pad, wide, style):
    _rope(eb, rows, hq, hkv, d, torch.float32, BF, norm, style, rot, sections, seed=rows, pad=pad, wide=wide)


def test_rope_far_and_negative_positions(eb):
    pos = A.ints([[0, 1, -1, -70000, 10 ** 6, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31]])
    _rope(eb, 8, 2, 2, 128, torch.float32, FP, None, "half", 128, (64,), pos=pos)


def test_rope_zero_head(eb):
    """A head of zeros stays zero under a norm with eps > 0."""
    cache = eb.empty_kv_cache(1, 16, 1, 64, BF)
    x = torch.zeros(2, 3 * 64, device=DEV)
    f = torch.ones(32, device=DEV)
    q = eb.rope_append(x, cache, A.ints([0, 1]), A.ints([3, 4]), f, 1, torch.ones(64, device=DEV),
                       torch.ones(64, device=DEV), 1e-6)
    assert bool((q == 0).all()) and bool((cache.k[0, 0, :2] == 0).all())


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def _attn(eb, seqs, hq, hkv, d, dtype, page=16, mask="causal", prefix=None, window=0, cap=0.0, seed=1,
          scale=None, pad=0, max_new=None, q_gain=1.5):
    """seqs: (new, kv) of each sequence."""
    new, lens = [n for n, _ in seqs], [t for _, t in seqs]
    k, v, table = A.paged(lens, page, hkv, d, dtype, seed)
    q = (_randn(sum(new) + pad, hq, d, seed=seed + 1) * q_gain).to(dtype)
    q_start, kv_len = A.starts(new), A.ints(lens)
    pre = A.ints(prefix) if prefix is not None else None
    out = torch.full_like(q, 7.0)
    mn = max_new or max(max(new), 1)
    got = eb.attention(q, eb.KVCache(k, v), table, q_start, kv_len, mn, max(max(lens), 1), mask, pre, window,
                       cap, scale, out=out)
    torch.cuda.synchronize()
    ref, err = A.attn_ref(q, k, v, table, q_start, kv_len, mask, prefix, window, cap, scale, mn)
    A.assert_attn(got, ref, err, str(seqs[:4]), untouched=7.0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (6, 2), (4, 4)])
def test_attn_decode_lengths(eb, d, dtype, hq, hkv):
    _attn(eb, [(1, t) for t in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300)], hq, hkv, d, dtype, seed=d)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("new,kv", [(2, 2), (33, 33), (31, 70), (64, 64), (65, 200), (129, 129), (150, 333)])
@pytest.mark.parametrize("mask", ["causal", "full"])
def test_attn_chunks(eb, d, dtype, new, kv, mask):
    _attn(eb, [(new, kv)], 4, 2, d, dtype, mask=mask, seed=new)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (7, 1), (33, 1), (48, 1), (10, 5), (64, 2), (200, 1)])
@pytest.mark.parametrize("new,kv", [(1, 77), (3, 77), (40, 90)])
def test_attn_groups(eb, hq, hkv, new, kv):
    _attn(eb, [(new, kv), (1, 5)], hq, hkv, 64, BF, seed=hq)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 4096])
def test_attn_pages(eb, page):
    _attn(eb, [(5, 100), (1, 16), (70, 257)], 4, 2, 128, BF, page=page, seed=page)


@pytest.mark.parametrize("mask,prefix,window,cap", [
    ("causal", [0, 20, 500, 3], 0, 0.0), ("causal", None, 1, 0.0), ("causal", None, 17, 0.0),
    ("causal", [40, 1, 64, 9], 33, 0.0), ("causal", None, 0, 5.0), ("full", None, 0, 30.0),
    ("full", None, 25, 0.0), ("causal", [50, 50, 50, 50], 64, 10.0), ("causal", None, 0, 2.0 ** -10),
    ("causal", None, 50, 1024.0)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_attn_masks(eb, mask, prefix, window, cap, d):
    _attn(eb, [(40, 130), (64, 64), (1, 200), (100, 300)], 4, 1, d, BF if d != 64 else FP, mask=mask,
          prefix=prefix, window=window, cap=cap, seed=window + 3)


# 64 query heads for each of 4: sequences whose 128-row tiles fill the GPU, which
# take the kernel that shares key tiles between four waves of rows
WIDE = dict(hq=256, hkv=4)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("mask,prefix,window,cap,kv", [
    ("causal", None, 0, 0.0, 130), ("causal", None, 0, 0.0, 423), ("full", None, 0, 0.0, 161),
    ("causal", [90], 0, 20.0, 200), ("causal", None, 21, 0.0, 300), ("full", None, 40, 5.0, 257)])
def test_attn_row_tiles(eb, d, dtype, mask, prefix, window, cap, kv):
    _attn(eb, [(130, kv)], d=d, dtype=dtype, mask=mask, prefix=prefix, window=window, cap=cap, seed=kv, **WIDE)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (128, 128), (256, 16), (256, 64)])
def test_attn_row_tiles_ragged(eb, d, page):
    """Tiles of many sequences, one of them long enough to be split; tokens past max_new,
    rows that see nothing, padding."""
    seqs = [(100, 100), (1, 40), (31, 500), (0, 7), (3, 2), (40, 3000), (2, 0), (15, 16)]
    _attn(eb, seqs, d=d, dtype=BF, page=page, seed=d + page, pad=4, **WIDE)
    _attn(eb, seqs, d=d, dtype=BF, page=page, seed=d + page, mask="full", max_new=37, hq=384, hkv=6)


def test_attn_row_tiles_many_sequences(eb):
    rng = np.random.default_rng(3)
    seqs = [(int(rng.integers(0, 6)), int(rng.integers(1, 60))) for _ in range(90)] + [(20, 2500), (7, 7)]
    _attn(eb, seqs, d=64, dtype=FP, seed=4, pad=2, **WIDE)


def test_attn_sharp_scores(eb):
    """Scores far apart, of both signs, a scale of one, a negative one and none."""
    for i, (gain, scale) in enumerate(((30.0, None), (4.0, 1.0), (2.0, -0.3), (1.0, 0.0))):
        _attn(eb, [(70, 300), (1, 1000)], 4, 2, 128, BF, seed=40 + i, q_gain=gain, scale=scale)


@pytest.mark.parametrize("batch", [2, 63, 64, 65, 130, 700])
def test_attn_many_sequences(eb, batch):
    rng = np.random.default_rng(batch)
    seqs = []
    for _ in range(batch):
        t = int(rng.integers(1, 90))
        n = 0 if rng.random() < 0.2 else 1 if rng.random() < 0.7 else int(rng.integers(1, t + 1))
        seqs.append((n, t))
    seqs[-1] = (1, 1500)
    _attn(eb, seqs, 2, 1, 64, BF, seed=batch, pad=5)


def test_attn_empty_rows_and_padding(eb):
    """No keys, no new tokens, more new tokens than keys, rows behind the last sequence."""
    _attn(eb, [(1, 0), (0, 40), (5, 3), (0, 0), (2, 2)], 4, 2, 64, BF, pad=3)
    _attn(eb, [(9, 4), (3, 0)], 4, 2, 128, FP, mask="full", pad=40)
    _attn(eb, [(50, 20)], 8, 1, 64, BF)
    _attn(eb, [(300, 100)], 1, 1, 64, BF, prefix=[7])
    _attn(eb, [(1, 0)], 1, 1, 64, BF)
    # tokens past max_new are not computed
    _attn(eb, [(40, 60), (7, 9), (130, 130)], 4, 2, 64, BF, max_new=5)
    _attn(eb, [(200, 260), (7, 9)], 2, 2, 64, BF, max_new=70)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 3e38])
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 2), (128, 4, 2), (256, 4, 2), (64, 256, 4), (128, 256, 4), (256, 256, 4)])
def test_attn_masked_places_hold_anything(eb, bad, d, hq, hkv):
    """Cache rows past a sequence's end, pages of nobody, keys and values that the causal
    mask, the window or the missing page hides."""
    new, lens, page = [37, 1, 100], [90, 33, 100], 16
    k, v, table = A.paged(lens, page, hkv, d, BF, seed=5)
    q = (_randn(138, hq, d, seed=6) * 1.5).to(BF)
    used = torch.zeros(k.shape[0] * page, dtype=torch.bool)
    for b, t in enumerate(lens):
        j = torch.arange(t)
        used[table[b].cpu().long()[j // page] * page + j % page] = True

    def spoil(c, cells):
        c = c.transpose(1, 2).contiguous()
        c.view(-1, hkv, d)[cells.to(DEV)] = bad
        return c.transpose(1, 2).contiguous()

    args = (table, A.starts(new), A.ints(lens), 100, 100)
    clean = eb.attention(q, eb.KVCache(k, v), *args)
    got = eb.attention(q, eb.KVCache(spoil(k, ~used), spoil(v, ~used)), *args)
    assert torch.equal(got, clean)
    ref, err = A.attn_ref(q, k, v, table, A.starts(new), A.ints(lens))
    A.assert_attn(clean, ref, err, "clean")
    # the last 20 tokens of sequence 2 spoiled: the rows before them do not see it
    j = torch.arange(80, 100)
    cells = torch.zeros_like(used)
    cells[table[2].cpu().long()[j // page] * page + j % page] = True
    got = eb.attention(q, eb.KVCache(spoil(k, cells), spoil(v, cells)), *args)
    A.assert_attn(got[:118], ref[:118], err[:118], "after the row")
    # the first 30 tokens of every sequence spoiled, hidden by a window of 20
    cells = torch.zeros_like(used)
    for b in (0, 2):
        j = torch.arange(30)
        cells[table[b].cpu().long()[j // page] * page + j % page] = True
    ks, vs = spoil(k, cells), spoil(v, cells)
    got = eb.attention(q, eb.KVCache(ks, vs), *args, window=20)
    refw, errw = A.attn_ref(q, k, v, table, A.starts(new), A.ints(lens), window=20)
    A.assert_attn(got[:38], refw[:38], errw[:38], "window")
    A.assert_attn(got[38 + 49:], refw[38 + 49:], errw[38 + 49:], "window")
    # a missing page hides the same tokens
    t2 = table.clone()
    t2[0, 0], t2[2, 0], t2[0, 1], t2[2, 1] = -1, k.shape[0], -2 ** 31, 2 ** 31 - 1
    got = eb.attention(q, eb.KVCache(ks, vs), t2, *args[1:])
    refm, errm = A.attn_ref(q, k, v, t2, A.starts(new), A.ints(lens))
    A.assert_attn(got, refm, errm, "missing page")


def test_attn_wild_lengths_stay_in_bounds(eb):
    """Offsets and lengths that are no such thing are clamped to their arrays."""
    k, v, table = A.paged([64, 64], 16, 2, 64, BF, seed=3)
    cache = eb.KVCache(k, v)
    for hq in (4, 1024):   # few rows, and 128-row tiles
        q = _randn(20, hq, 64, seed=4, dtype=BF)
        for q_start in ([0, 10, 2 ** 31 - 1], [-5, 10, 20], [15, 3, 20], [0, 2 ** 31 - 1, -2 ** 31], [20, 25, 30]):
            for kv in ([2 ** 31 - 1, 64], [-3, -2 ** 31]):
                for pre in (None, [2 ** 31 - 1, -2 ** 31]):
                    out = torch.full_like(q, 7.0)
                    eb.attention(q, cache, table, A.ints(q_start), A.ints(kv), 20, 64, out=out,
                                 prefix=None if pre is None else A.ints(pre))
                    assert bool(torch.isfinite(out).all())
    # many sequences that all claim all rows: more tiles than there can be
    q = _randn(200, 32, 64, seed=4, dtype=BF)
    batch = 600
    many = table[:1].repeat(batch, 1)
    out = torch.full_like(q, 7.0)
    eb.attention(q, cache, many, A.ints([0, 200] * (batch // 2) + [0]), A.ints([64] * batch), 200, 64, out=out)
    assert bool(torch.isfinite(out).all())


def test_attn_strided_rows_and_scratch(eb):
    """Queries and outputs as columns of wider buffers; a workspace of the caller's."""
    k, v, table = A.paged([200, 50], 32, 2, 64, FP, seed=8)
    cache = eb.KVCache(k, v)
    new, lens = [1, 30], [200, 50]
    wide = _randn(31, 4 * 64 + 40, seed=9, dtype=FP)
    q = wide[:, 8:8 + 256].unflatten(1, (4, 64))
    buf = torch.full((31, 4 * 64 + 24), 7.0, dtype=FP, device=DEV)
    out = buf[:, 16:16 + 256].unflatten(1, (4, 64))
    n = eb.attention_workspace_bytes((31, 4, 64), cache, 2, table.shape[1], 30, 200)
    ws = torch.full((max(n, 1),), 255, dtype=torch.uint8, device=DEV)  # NaN, to begin with
    eb.attention(q, cache, table, A.starts(new), A.ints(lens), 30, 200, out=out, workspace=ws)
    ref, err = A.attn_ref(q.contiguous(), k, v, table, A.starts(new), A.ints(lens))
    A.assert_attn(out.contiguous(), ref, err, "strided")
    assert bool((buf[:, :16] == 7.0).all()) and bool((buf[:, 272:] == 7.0).all())


def test_attn_same_bits_twice(eb):
    k, v, table = A.paged([3000, 700], 16, 2, 128, BF, seed=8)
    q = _randn(41, 8, 128, seed=9, dtype=BF)
    args = (eb.KVCache(k, v), table, A.starts([1, 40]), A.ints([3000, 700]), 40, 3000)
    first = eb.attention(q, *args)
    for _ in range(4):
        assert torch.equal(eb.attention(q, *args), first)


def test_attn_offsets_past_32_bits(eb):
    """Pages behind 2^31 elements and 2^32 bytes of the cache."""
    heads, page, d = 8, 256, 128
    pages = 2 ** 31 // (heads * page * d) + 40
    k = torch.empty(pages, heads, page, d, dtype=BF, device=DEV)
    v = torch.empty(pages, heads, page, d, dtype=BF, device=DEV)
    ids = [pages - 1, 3, pages - 30]
    small_k, small_v = _randn(3, heads, page, d, seed=1, dtype=BF), _randn(3, heads, page, d, seed=2, dtype=BF)
    for i, p in enumerate(ids):
        k[p], v[p] = small_k[i], small_v[i]
    new, lens = [40], [700]
    q = _randn(40, 16, d, seed=3, dtype=BF)
    cache = eb.KVCache(k, v)
    got = eb.attention(q, cache, A.ints([ids]), A.starts(new), A.ints(lens), 40, 700)
    one = eb.attention(q[-1:].contiguous(), cache, A.ints([ids]), A.starts([1]), A.ints(lens), 1, 700)
    ref, err = A.attn_ref(q, small_k, small_v, A.ints([[0, 1, 2]]), A.starts(new), A.ints(lens))
    A.assert_attn(got, ref, err, "far pages")
    A.assert_attn(one, ref[-1:], err[-1:], "far pages, one token")
    x = _randn(2, (16 + 2 * heads) * d, seed=5)
    slots = [(pages - 1) * page + 255, (pages - 20) * page]
    eb.rope_append(x, cache, A.ints(slots), None, None, 16)
    for r, s in enumerate(slots):
        want = x[r].view(-1, d)[16:].to(BF)
        assert torch.equal(k[s // page, :, s % page], want[:heads])
        assert torch.equal(v[s // page, :, s % page], want[heads:])


# ---------------------------------------------------------------------------
# together: a layer's steps, prompts and then tokens one by one
# ---------------------------------------------------------------------------

class _Layer:
    """QKV -> rope_append -> attention -> O + h of one layer over a growing batch."""

    def __init__(self, eb, dm, hq, hkv, d, qtype, dtype, seed):
        self.eb, self.hq, self.hkv, self.d, self.dtype = eb, hq, hkv, d, dtype
        self.wqkv = W.normal(((hq + 2 * hkv) * d, dm), seed, DEV, 0.05)
        self.wo = W.normal((dm, hq * d), seed + 1, DEV, 0.05)
        self.qkv, self.o = eb.quantize(self.wqkv, qtype), eb.quantize(self.wo, qtype)
        self.gamma = 1 + 0.1 * W.normal((dm,), seed + 2, DEV)
        self.gq = 1 + 0.1 * W.normal((d,), seed + 3, DEV)
        self.gk = 1 + 0.1 * W.normal((d,), seed + 4, DEV)
        self.freqs = (1e4 ** (-torch.arange(d // 2) / (d // 2))).float().to(DEV)
        self.cache = eb.empty_kv_cache(40, 16, hkv, d, dtype)
        self.cache.k.fill_(float("nan"))
        self.cache.v.fill_(float("nan"))

    def step(self, h, b, table, max_new, max_kv):
        eb = self.eb
        qkv = eb.qlinear_fused(self.qkv, h, x_dtype=self.dtype, prologue="rmsnorm", norm_weight=self.gamma,
                               eps=1e-5)
        q = eb.rope_append(qkv, self.cache, b.slots, b.positions, self.freqs, self.hq, self.gq, self.gk, 1e-6)
        o = torch.zeros_like(q)   # the O projection reads padding rows too
        eb.attention(q, self.cache, table, b.q_start, b.kv_len, max_new, max_kv, out=o)
        return eb.qlinear_fused(self.o, o.flatten(1), epilogue="add", residual=h)


@pytest.mark.parametrize("dtype,qtype", [(BF, "q8_0"), (FP, "q4_0")])
def test_layer_prompts_then_tokens(eb, dtype, qtype):
    """Prompts in chunks, then tokens one by one, in a batch: each token's output equals the
    one of its whole sequence run as one prompt, to the rounding of weights and outputs."""
    dm, hq, hkv, d, page = 256, 4, 2, 64, 16
    total = [61, 20, 97]
    L = _Layer(eb, dm, hq, hkv, d, qtype, dtype, 50)
    hs = [W.normal((t, dm), 70 + i, DEV) for i, t in enumerate(total)]
    free, n_free = A.ints(np.random.default_rng(0).permutation(40)), A.ints([40])
    table = torch.full((3, 8), -1, dtype=torch.int32, device=DEV)
    done, outs = [0, 0, 0], [[], [], []]
    steps = [[30, 0, 64], [11, 5, 20]] + [[1, 1, 1]] * 12 + [[8, 2, 1], [0, 1, 0]]
    for add in steps:
        add = [min(a, total[i] - done[i]) for i, a in enumerate(add)]
        b = eb.kv_extend(table, A.ints(done), A.ints(add), free, n_free, page, 40, sum(add) + 2)
        n_free = b.n_free
        h = torch.cat([hs[i][done[i]:done[i] + a] for i, a in enumerate(add)] + [torch.ones(2, dm, device=DEV)])
        y = L.step(h, b, table, max(add), 128)
        at = 0
        for i, a in enumerate(add):
            outs[i].append(y[at:at + a])
            at += a
            done[i] += a
        assert int(b.short) == 0 and b.kv_len.tolist() == done
    assert done == total
    assert int(n_free) == 40 - sum(-(-t // page) for t in total)
    # whole sequences at once, on fresh pages
    table2 = torch.full((3, 8), -1, dtype=torch.int32, device=DEV)
    b = eb.kv_extend(table2, A.ints([0, 0, 0]), A.ints(total), free, A.ints([40]), page, 40, sum(total))
    want = L.step(torch.cat(hs), b, table2, max(total), 128)
    got = torch.cat([torch.cat(o) for o in outs])
    # Both sides round attention's weights and outputs by up to u each, spread about 0.6 u
    # of values of 0.8 (a normed row of 256 times weights of 0.05); the O projection adds 256
    # such differences times 0.05: 0.4 u spread, 2 u at 4.5 of it on 45000 outputs.  8 u
    # leaves room for queries, keys and values that round to neighbours on the two sides.
    assert float((got - want).abs().max()) <= 8 * A.HALF_ULP[dtype]


def test_step_captured_and_replayed(eb):
    """A decode step captured once and replayed as the lengths grow, beside eager work on
    another stream, equals the eager step; two graphs have a workspace each."""
    dm, hq, hkv, d, page, batch = 256, 8, 2, 64, 16, 3
    L = _Layer(eb, dm, hq, hkv, d, "q8_0", BF, 90)
    L.cache.k.copy_(_randn(*L.cache.k.shape, seed=1))
    L.cache.v.copy_(_randn(*L.cache.v.shape, seed=2))
    have = [300, 17, 1]
    lists = A.ints(np.random.default_rng(1).permutation(40))
    table = torch.full((batch, 24), -1, dtype=torch.int32, device=DEV)
    first = eb.kv_extend(table, A.ints([0] * 3), A.ints(have), lists, A.ints([40]), page, 40, sum(have))
    cached, n_free = first.kv_len.clone(), first.n_free.clone()
    added = A.ints([1, 1, 1])
    h = W.normal((batch + 1, dm), 91, DEV)

    def step():
        b = eb.kv_extend(table, cached, added, lists, n_free, page, 40, batch + 1)
        y = L.step(h, b, table, 1, 384)
        return b, y

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()   # nothing is lost: the same pages are taken again
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b, y = step()
        graphs.append((g, b, y))
    for it in range(20):
        b0, y0 = step()
        want = (y0.clone(), b0.slots.clone(), table.clone())
        for g, b, y in graphs:
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want[0]) and torch.equal(b.slots, want[1]) and torch.equal(table, want[2]), it
        cached.copy_(b0.kv_len)
        n_free.copy_(b0.n_free)
        h.copy_(torch.roll(h, 1, 0) * 0.9 + 0.1)
    # both graphs at once on two streams: neither disturbs the other
    _, y0 = step()
    want = y0.clone()
    s2 = torch.cuda.Stream()
    torch.cuda.synchronize()
    for g, _, y in graphs:
        y.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        graphs[0][0].replay()
        with torch.cuda.stream(s2):
            graphs[1][0].replay()
    torch.cuda.synchronize()
    for _, _, y in graphs:
        assert torch.equal(y, want)


def test_large_batch_captured(eb):
    """A batch whose items a kernel lays out first, captured and replayed as lengths change."""
    batch = 130
    lens = [int(t) for t in np.random.default_rng(5).integers(1, 300, batch)]
    k, v, table = A.paged(lens, 16, 1, 64, BF, seed=6)
    cache = eb.KVCache(k, v)
    q = _randn(batch, 8, 64, seed=7, dtype=BF)
    q_start, kv_len = A.starts([1] * batch), A.ints(lens)
    args = (cache, table, q_start, kv_len, 1, 300)
    eb.attention(q, *args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = eb.attention(q, *args)
    for it in range(4):
        want = eb.attention(q, *args).clone()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), it
        kv_len.copy_((kv_len * 3 // 4).clamp(min=1))


def test_other_stream(eb):
    """Calls on a side stream take their workspace from that stream."""
    k, v, table = A.paged([900], 16, 1, 64, BF, seed=8)
    q = _randn(1, 8, 64, seed=9, dtype=BF)
    args = (eb.KVCache(k, v), table, A.starts([1]), A.ints([900]), 1, 900)
    want = eb.attention(q, *args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [eb.attention(q, *args) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(g, want) for g in got)


# One sequence, and batches, whose keys are split between workgroups: max_new and max_kv
# bound more than is there, as in a captured graph, and the kernel, its tiles and the
# number of splits follow from them.
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("seqs,hq,hkv,max_new,max_kv,mask,prefix,window,cap", [
    ([(40, 2600)], 8, 2, 40, 16000, "causal", None, 0, 0.0),
    ([(40, 2600)], 8, 1, 300, 60000, "full", None, 0, 20.0),
    ([(130, 1500)], 8, 1, 130, 16000, "causal", None, 0, 0.0),
    ([(60, 1100)], 32, 8, 300, 16000, "causal", None, 0, 0.0),
    ([(60, 1111)], 32, 8, 600, 64000, "causal", [1090], 0, 5.0),
    ([(90, 1100)], 16, 2, 600, 64000, "causal", None, 900, 0.0),
    ([(33, 700)], 64, 8, 50, 100000, "full", None, 0, 0.0),
    ([(30, 1500), (1, 2500), (0, 9), (7, 40)], 16, 8, 30, 16000, "causal", None, 0, 0.0),
    ([(40, 300), (9, 9), (1, 1100), (13, 800), (2, 2)], 32, 8, 40, 16000, "causal", [0, 3, 0, 795, 1], 0, 0.0),
    ([(1, 30)] * 40 + [(3, 3000), (0, 4)] + [(5, 20)] * 30, 8, 2, 40, 60000, "causal", None, 0, 0.0),
    ([(1, 16)] * 69 + [(1, 9000)], 8, 2, 1, 60000, "causal", None, 0, 0.0)])
def test_attn_splits(eb, d, seqs, hq, hkv, max_new, max_kv, mask, prefix, window, cap):
    new, lens = [n for n, _ in seqs], [t for _, t in seqs]
    k, v, table = A.paged(lens, 16, hkv, d, BF, seed=d)
    q = (_randn(sum(new) + 3, hq, d, seed=d + 1) * 1.5).to(BF)
    q_start, kv_len = A.starts(new), A.ints(lens)
    pre = A.ints(prefix) if prefix is not None else None
    out = torch.full_like(q, 7.0)
    eb.attention(q, eb.KVCache(k, v), table, q_start, kv_len, max_new, max_kv, mask, pre, window, cap, out=out)
    torch.cuda.synchronize()
    ref, err = A.attn_ref(q, k, v, table, q_start, kv_len, mask, prefix, window, cap)
    A.assert_attn(out, ref, err, str(seqs[:4]), untouched=7.0)


@pytest.mark.parametrize("d,hq,hkv,max_new,max_kv", [
    (64, 8, 1, 40, 16000), (128, 8, 1, 40, 16000), (256, 8, 1, 40, 16000), (64, 32, 8, 300, 16000),
    (128, 32, 8, 300, 16000), (256, 32, 8, 600, 64000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attn_splits_masked_places_hold_anything(eb, d, hq, hkv, max_new, max_kv, bad):
    """The last 20 places of one sequence hold no numbers: tokens before them see none of it."""
    new, kv = 40, 1100
    k, v, table = A.paged([kv], 16, hkv, d, BF, seed=d)
    for p in range(kv - 20, kv):
        page = int(table[0, p // 16])
        k[page, :, p % 16] = bad
        v[page, :, p % 16] = bad
    q = _randn(new, hq, d, seed=d + 1).to(BF)
    q_start, kv_len = A.starts([new]), A.ints([kv])
    out = eb.attention(q, eb.KVCache(k, v), table, q_start, kv_len, max_new, max_kv)
    ref, err = A.attn_ref(q, k, v, table, q_start, kv_len)
    assert bool(torch.isnan(ref[20:]).all()) and bool(torch.isfinite(ref[:20]).all())
    A.assert_attn(out, ref, err, "before the last 20 places")
    assert not bool(torch.isfinite(out[20:].float()).any())


def test_attn_workspace_of_each_mask(eb):
    """Calls of the same sizes under other masks and windows, in either order: each takes
    the workspace that it needs, its own or the caller's."""
    kinds = [("causal", None, 100), ("causal", None, 0), ("full", None, 0), ("causal", [30], 0), ("full", None, 64),
             ("causal", [30], 100)]
    for order in (kinds, kinds[::-1]):
        eb._ATTN_WS_BYTES.clear()
        k, v, table = A.paged([300], 16, 2, 128, BF, seed=3)
        cache, q = eb.KVCache(k, v), _randn(40, 8, 128, seed=4).to(BF)
        q_start, kv_len = A.starts([40]), A.ints([300])
        needs = set()
        for mask, prefix, window in order:
            pre = A.ints(prefix) if prefix else None
            got = eb.attention(q, cache, table, q_start, kv_len, 40, 16000, mask, pre, window)
            n = eb.attention_workspace_bytes(q.shape, cache, 1, table.shape[1], 40, 16000, mask, pre is not None,
                                             window)
            needs.add(n)
            ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
            again = eb.attention(q, cache, table, q_start, kv_len, 40, 16000, mask, pre, window, workspace=ws)
            ref, err = A.attn_ref(q, k, v, table, q_start, kv_len, mask, prefix, window)
            A.assert_attn(got, ref, err, f"{mask} {prefix} {window}")
            assert torch.equal(got, again)
        assert 0 in needs and len(needs) > 1
