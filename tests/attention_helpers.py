"""Plain references, in 64 bits on the CPU, of the steps between a layer's QKV
and O projections, and the error bounds of the GPU's (test infrastructure)."""
import numpy as np
import torch

HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def extend_ref(table, cached, added, free_pages, n_free, page, pages, rows):
    """Token by token; numpy int64 arrays in, a dict of what eb_kv_extend writes out."""
    table = table.copy()
    batch, stride = table.shape
    capacity = stride * page
    n_free = min(max(int(n_free), 0), len(free_pages))
    used = row = short = 0
    slots, positions = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    q_start, kv_len = [0], []
    for b in range(batch):
        have, new = max(int(cached[b]), 0), max(int(added[b]), 0)
        for p in range(have, have + new):
            slot = -1
            if p < capacity:
                fresh = p // page >= -(-have // page)
                if fresh and p % page == 0:
                    entry = int(free_pages[n_free - 1 - used]) if used < n_free else -1
                    entry = entry if 0 <= entry < pages else -1
                    used += 1
                    page_id = entry
                    if row < rows:
                        table[b, p // page] = entry
                elif not fresh:
                    page_id = int(table[b, p // page])
                if 0 <= page_id < pages:
                    slot = page_id * page + p % page
                else:
                    short += 1
            else:
                short += 1
            if row < rows:
                slots[row], positions[row] = slot, p
            row += 1
        q_start.append(min(row, rows))
        kv_len.append(min(have + new, capacity))
    return dict(table=table, q_start=q_start, kv_len=kv_len, slots=slots, positions=positions,
                n_free=[max(n_free - used, 0)], short=[short])


def rope_ref(x, hq, hkv, d, pos, freqs, style, sections, q_norm, k_norm, eps):
    """x [rows, (hq + 2 hkv) d] -> (q, k, v, scale of q, scale of k): float64, the scales
    being |a| + |b| of the pair that an output element comes from."""
    x = x.double().cpu().view(x.shape[0], hq + 2 * hkv, d)
    half = freqs.numel() if freqs is not None else 0

    def head(h, g):
        if g is not None:
            h = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * g.double().cpu()
        out, scale = h.clone(), h.abs()
        if half:
            axis = [a for a, n in enumerate(sections) for _ in range(n)]
            ang = (pos.view(-1, x.shape[0])[axis].double().cpu().T * freqs.double().cpu())[:, None]
            i = torch.arange(half)
            ia, ib = (i, i + half) if style == "half" else (2 * i, 2 * i + 1)
            a, b = h[..., ia], h[..., ib]
            out[..., ia] = a * torch.cos(ang) - b * torch.sin(ang)
            out[..., ib] = b * torch.cos(ang) + a * torch.sin(ang)
            scale[..., ia] = scale[..., ib] = a.abs() + b.abs()
        return out, scale

    q, sq = head(x[:, :hq], q_norm)
    k, sk = head(x[:, hq:hq + hkv], k_norm)
    return q, k, x[:, hq + hkv:], sq, sk


def assert_rope(got, ref, scale, what):
    """One rounding of the output, and before it: sums of up to 256 squares in a tree
    of at most 13 additions, a division, a root and products (under 24 half steps of
    fp32, 1.5e-6), and sines and cosines off by 5e-7: 2^-19 of |a| + |b| in all.  A
    binary16 result below its normal range rounds by 2^-25 whatever its size."""
    u = HALF_ULP[got.dtype]
    err = 2.0 ** -19 * scale
    tol = err + u * (ref.abs() + err) + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    bad = (got.double().cpu() - ref).abs() - tol
    assert float(bad.max()) <= 0, f"{what}: over the bound by {float(bad.max()):.3e}"


def seen(p, kv, mask, prefix, window):
    hi = kv if mask == "full" else min(kv, max(p + 1, prefix))
    return (max(0, p - window + 1) if window else 0), hi


def attn_ref(q, k, v, table, q_start, kv_len, mask="causal", prefix=None, window=0, softcap=0.0,
             scale=None, max_new=1 << 30):
    """Row by row and head by head: (out, err) in float64, NaN in `out` where a row is
    not written; err bounds the GPU's error before the output's rounding."""
    rows, hq, d = q.shape
    pages, hkv, page, _ = k.shape
    u = HALF_ULP[q.dtype]
    scale = d ** -0.5 if scale is None else scale
    qd, table = q.double().cpu(), table.cpu().long()
    out, err = torch.full(q.shape, float("nan"), dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    q_start, kv_len = q_start.cpu().tolist(), kv_len.cpu().tolist()
    group = hq // hkv
    for b in range(len(kv_len)):
        q0, q1 = q_start[b], min(q_start[b + 1], rows)
        kv = min(max(kv_len[b], 0), table.shape[1] * page)
        j = torch.arange(kv)
        ids = table[b, j // page]
        there = (ids >= 0) & (ids < pages)
        ids = ids.clamp(0, pages - 1)
        kb = k.cpu()[ids, :, j % page].double()   # [kv, hkv, d]
        vb = v.cpu()[ids, :, j % page].double()
        for r in range(q0, min(q1, q0 + max_new)):
            p = kv - (q1 - q0) + r - q0
            lo, hi = seen(p, kv, mask, int(prefix[b]) if prefix is not None else 0, window)
            keep = torch.zeros(kv, dtype=torch.bool)
            keep[lo:max(lo, hi)] = True
            keep &= there
            if not bool(keep.any()):
                out[r] = 0
                continue
            kk, vv = kb[keep].transpose(0, 1), vb[keep].transpose(0, 1)   # [hkv, n, d]
            qq = qd[r].view(hkv, group, d)
            t = qq @ kk.transpose(1, 2) * scale
            size = (qq.abs() @ kk.abs().transpose(1, 2) * abs(scale)).amax(-1, keepdim=True)
            if softcap:
                t = softcap * torch.tanh(t / softcap)
            w = torch.softmax(t, -1)
            out[r] = (w @ vv).reshape(hq, d)
            # scores: d fp32 additions of exact products and three roundings of the scaled
            # sum; the cap's tanh to 2^-21 of the cap; 2^t to 2^-21; weights rounded to u in
            # the numerator, not in the sum; sums of n weights, 16 at a time
            delta = size * (d + 4) * 2.0 ** -24 + (softcap * 2.0 ** -20 if softcap else 0.0) + 2.0 ** -21
            e = u + 2 * delta + 2 * (int(keep.sum()) / 16 + 64) * 2.0 ** -24
            err[r] = ((w @ vv.abs()) * e).reshape(hq, d)
    return out, err


def assert_attn(got, ref, err, what, untouched=None):
    u = HALF_ULP[got.dtype]
    got = got.double().cpu()
    live = ~torch.isnan(ref)
    tol = err + u * (ref.abs() + err) + (2.0 ** -25 if u == 2.0 ** -11 else 0.0)
    bad = ((got - ref).abs() - tol)[live]
    assert bool(torch.isfinite(got[live]).all()), f"{what}: not finite"
    if bad.numel():
        assert float(bad.max()) <= 0, f"{what}: over the bound by {float(bad.max()):.3e}"
    if untouched is not None:
        assert bool((got[~live] == untouched).all()), f"{what}: a row that is not computed was written"


def paged(lens, page, heads, d, dtype, seed, spare=3, stride=None, device="cuda"):
    """A cache of random values, a block table of shuffled pages and its used part."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    held = [-(-t // page) for t in lens]
    pages = sum(held) + spare
    order = rng.permutation(pages)
    stride = stride or max(1, max(held))
    table, at = np.full((len(lens), stride), -1, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    k = torch.randn(pages, heads, page, d, generator=g).to(dtype).to(device)
    v = torch.randn(pages, heads, page, d, generator=g).to(dtype).to(device)
    return k, v, torch.from_numpy(table).to(device)


def ints(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32).to(device)


def starts(new, device="cuda"):
    return ints(np.concatenate([[0], np.cumsum(new)]), device)
