"""A plain reference of eb_kv_extend, token by token, for steps of any number of rows
(test infrastructure)."""
import numpy as np


def extend_ref(table, cached, added, free_pages, n_free, page, pages, rows):
    """numpy int64 arrays in, a dict of what eb_kv_extend writes out.  The batch's first
    `rows` new tokens join; the others take nothing and count as short."""
    table, (batch, stride) = table.copy(), table.shape
    stack = [int(p) for p in free_pages[:min(max(int(n_free), 0), len(free_pages))]]
    slots, positions = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    q_start, kv_len, row, short = [0], [], 0, 0
    for b in range(batch):
        have, new = max(int(cached[b]), 0), max(int(added[b]), 0)
        joined = min(new, rows - row)
        short += new - joined
        held = -(-have // page)
        for p in range(have, have + joined):
            entry = -1
            if p < stride * page:
                if p // page >= held and p % page == 0:
                    entry = stack.pop() if stack else -1
                    table[b, p // page] = entry if 0 <= entry < pages else -1
                entry = int(table[b, p // page])
                entry = entry if 0 <= entry < pages else -1
            slots[row] = entry * page + p % page if entry >= 0 else -1
            positions[row] = p
            short += entry < 0
            row += 1
        q_start.append(row)
        kv_len.append(min(have + joined, stride * page))
    return dict(table=table, q_start=q_start, kv_len=kv_len, slots=slots, positions=positions,
                n_free=[len(stack)], short=[min(short, 2 ** 31 - 1)])


def extend_case(lens, page, seed, spare=2, stride=None, rows=None, n_free=None):
    """lens: (cached, added); pages in shuffled order, a table of entries that are no pages
    behind the held ones, and a step of `rows` rows (by default one for each token)."""
    rng = np.random.default_rng(seed)
    held = [-(-max(c, 0) // page) for c, _ in lens]
    total = [-(-(max(c, 0) + max(a, 0)) // page) for c, a in lens]
    pages = sum(total) + spare
    order = rng.permutation(pages).astype(np.int32)
    stride = stride or max(1, max(total))
    table, at = np.full((len(lens), stride), -7, np.int32), 0
    for b, h in enumerate(held):
        table[b, :min(h, stride)] = order[at:at + h][:stride]
        at += h
    free = order[at:]
    if rows is None:
        rows = sum(max(a, 0) for _, a in lens)
    return dict(table=table, cached=np.array([c for c, _ in lens]), added=np.array([a for _, a in lens]),
                free=free, n_free=len(free) if n_free is None else n_free, page=page, pages=pages, rows=rows)
