"""Definition of the page pool, one sequence and one page at a time: plain Python on lists; shares nothing with the device code."""


def resize(ring, state, table, old, new, page):
    """-> (ring, state, table, cu, positions, slots) after taking sequences from `old` to `new` tokens."""
    n, wide = len(ring), len(table[0]) if table else 1
    ring, table = list(ring), [list(r) for r in table]
    first, free = state[0] % 2 ** 32 % n, min(max(state[1], 0), n)
    before = list(ring)
    wanted, back, cu, positions, slots = 0, [], [0], [], []
    for row, o, w in zip(table, old, new):
        o, w = max(o, 0), max(w, 0)
        p0, p1 = min(-(-o // page), wide), min(-(-w // page), wide)
        back += [x for x in row[p1:p0] if 0 <= x < n]
        for entry in range(p0, p1):
            row[entry] = before[(first + wanted) % n] if wanted < free else -1
            wanted += 1
        for pos in range(o, w):
            p = row[pos // page] if pos // page < wide else -1
            positions.append(pos)
            slots.append(p * page + pos % page if 0 <= p < n else -1)
        cu.append(min(cu[-1] + max(w - o, 0), 2 ** 31 - 1))
    used, kept = min(wanted, free), back[:n - free]
    for i, x in enumerate(kept):
        ring[(first + free + i) % n] = x
    return ring, [(first + used) % n, free - used + len(kept), wanted - used, 0], table, cu, positions, slots
