"""The pages of a cache by the rules that include/heal.h gives, one entry after another."""


def held_blocks(n, block):
    return -(-max(n, 0) // block)


def release(table, refs, lens, block):
    for row, n in zip(table, lens):
        for b in range(held_blocks(n, block), len(row)):
            if 0 <= row[b] < len(refs):
                refs[row[b]] -= 1
            row[b] = -1


def fork(table, refs, lens, parents, children, block):
    before = [list(row) for row in table]
    for j, (p, c) in enumerate(zip(parents, children)):
        if not (0 <= p < len(table) and 0 <= c < len(table)) or c in parents or c in children[:j]:
            continue
        for b, old in enumerate(table[c]):
            new = before[p][b] if b < held_blocks(lens[p], block) else -1
            if not 0 <= new < len(refs):
                new = -1
            if 0 <= old < len(refs):
                refs[old] -= 1
            if new >= 0:
                refs[new] += 1
            table[c][b] = new


def touched(cu, lens, cols, block):
    """(row, block) of every entry that the new tokens touch, in order."""
    out = []
    for i, n in enumerate(lens):
        new = cu[i + 1] - cu[i]
        if new > 0 and n > 0:
            out += [(i, b) for b in range(max(n - new, 0) // block, (n - 1) // block + 1) if b < cols]
    return out


def reserve(table, refs, lens, cu, block):
    """Returns what lacks."""
    units = touched(cu, lens, len(table[0]) if table else 0, block)
    was, here = list(refs), {}
    for i, b in units:
        here.setdefault(table[i][b], []).append((i, b))

    def keeps(i, b):
        page = table[i][b]
        return 0 <= page < len(refs) and was[page] >= 1 and len(here[page]) >= was[page] and here[page][0] == (i, b)
    take = [u for u in units if not keeps(*u)]
    free = [p for p, r in enumerate(was) if r <= 0]
    if len(take) > len(free):
        return len(take) - len(free)
    for page, who in here.items():
        if 0 <= page < len(refs) and was[page] >= 1:
            refs[page] = 1 if len(who) >= was[page] else was[page] - len(who)
    for (i, b), page in zip(take, free):
        table[i][b], refs[page] = page, 1
    return 0


def compact(table, refs):
    """Returns the moves, [(src, dst)]."""
    moves, lo, hi = [], 0, len(refs) - 1
    while True:
        while lo < len(refs) and refs[lo] > 0:
            lo += 1
        while hi >= 0 and refs[hi] <= 0:
            hi -= 1
        if lo > hi:
            break
        refs[lo], refs[hi] = refs[hi], 0
        moves.append((hi, lo))
    to = dict(moves)
    for row in table:
        row[:] = [to.get(p, p) for p in row]
    return moves
