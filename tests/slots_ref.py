"""kv_slots as a loop over sequences and tokens."""
import numpy as np

PAGE = 16


def slots(table, held, added, rows, first=None, free=None, used=0):
    """(slots, positions, token_ptr, held afterwards, used afterwards, table afterwards)."""
    table = table.copy()
    width, at, take = table.shape[1], 0, max(0, used)
    out, pos, ptr, after = [-1] * rows, [0] * rows, [0], []
    for r, h in enumerate(held):
        h = max(0, int(h))
        n = 1 if added is None else min(max(0, int(added[r])), 2 ** 31 - 1 - h)
        n = min(n, rows - at)
        had, room = -(-h // PAGE), -(-h // PAGE)
        if free is None:
            room = width
        else:
            while room < min(-(-(h + n) // PAGE), width) and take < len(free):
                table[r, room] = free[take]
                take += 1
                room += 1
        for x in range(h, h + n):
            j = x // PAGE
            if j < min(room, width) and 0 <= table[r, j] <= (2 ** 31 - 1) // PAGE:
                out[at] = int(table[r, j]) * PAGE + x % PAGE
            pos[at] = x + (0 if first is None else int(first[r]))
            at += 1
        after.append(h + min(n, max(0, min(room, width) * PAGE - h)))
        ptr.append(at)
        del had
    return (np.array(out, np.int64), np.array(pos, np.int64), np.array(ptr), np.array(after),
            take if free is not None else None, table)
