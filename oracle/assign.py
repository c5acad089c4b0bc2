"""Oracle of handing out a cache's pages, one sequence and one page at a time, from the definition in
include/eb.h."""
from __future__ import annotations

import numpy as np


def assign(table, ring, state, cached, new, page_size, n_rows, done=None, shared=None):
    """Everything that a call writes, as a dict (table and ring: copies)."""
    table, ring = table.copy(), ring.copy()
    batch, wide = table.shape
    n_pages = len(ring)
    head, free = int(state[0]), int(state[1])
    demand = taken = back = 0
    cu_block, cu_prefix, pos, slot = [0], [0], [], []
    short = np.zeros(batch, np.uint8)
    for b in range(batch):
        held = -(-int(cached[b]) // page_size)
        if done is not None and done[b]:
            for j in range(0 if shared is None else int(shared[b]), held):
                ring[(head + free + back) % n_pages] = table[b, j]
                back += 1
            cu_block.append(cu_block[-1])
            cu_prefix.append(cu_prefix[-1])
            continue
        end = -(-(int(cached[b]) + int(new[b])) // page_size)
        placed = end <= wide
        if placed and end > held:
            demand += end - held
            placed = demand <= free
        for j in range(held, min(end, wide)):
            table[b, j] = ring[(head + taken + j - held) % n_pages] if placed else -1
        taken += end - held if placed else 0
        short[b] = not placed
        for p in range(int(cached[b]), int(cached[b]) + int(new[b])):
            number = table[b, p // page_size] if placed else -1
            pos.append(p if placed else -1)
            slot.append(int(number) * page_size + p % page_size if 0 <= number < n_pages else -1)
        cu_block.append(cu_block[-1] + int(new[b]))
        cu_prefix.append(cu_prefix[-1] + int(cached[b]))
    pad = [-1] * (n_rows - len(pos))
    return dict(table=table, ring=ring,
                state=np.array([(head + taken) % n_pages, free - taken + back], np.int32),
                cu_block=np.array(cu_block, np.int32), cu_prefix=np.array(cu_prefix, np.int32),
                pos=np.array(pos + pad, np.int32), slot=np.array(slot + pad, np.int64), short=short)
