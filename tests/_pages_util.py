"""Plain forms of the page planners, on lists (not collected by pytest)."""


def fork(table, lengths, parent, room, pages, P):
    """include/rrs.h, rrs_kv_fork: a dict of lists."""
    S, C = len(table), len(table[0])

    def pages_of(n):
        return -(-n // P)
    kept, want, old = [], [], []
    for b in range(S):
        p = b if parent is None else parent[b]
        if not 0 <= p < S:
            kept.append(0), want.append(0), old.append([])
            continue
        n = min(max(lengths[p], 0), C * P)
        want.append(min(max(room[b], 0), C * P))
        kept.append(min(n, want[b]))
        old.append(table[p][:pages_of(kept[b])])
    names = {}   # page -> rows that keep it, once per entry
    for b in range(S):
        for page in old[b]:
            if 0 <= page < pages:
                names.setdefault(page, []).append(b)

    def writes(b):
        return want[b] > kept[b] and kept[b] % P != 0 and 0 <= old[b][-1] < pages
    free = [p for p in range(pages) if p not in names]

    def plan(first_stays):
        copy, need = [], []
        for b in range(S):
            page = old[b][-1] if writes(b) else -1
            shared = writes(b) and len(names[page]) > 1
            if shared and first_stays:
                rows = [r for r in range(S) if writes(r) and old[r][-1] == page]
                shared = not (len(rows) == len(names[page]) and rows[0] == b)
            copy.append(shared)
            need.append(pages_of(want[b]) - len(old[b]) + shared)
        return copy, need
    copy, need = plan(True)
    if sum(need) > len(free):
        copy, need = plan(False)
    out, src, dst, got, upto, taken = [], [], [], [], 0, 0
    for b in range(S):
        row = list(old[b])
        begin, upto = upto, upto + need[b]
        if need[b] == 0 or upto <= len(free):
            fresh = free[begin:upto]
            taken += need[b]
            if copy[b]:
                src.append(row[-1]), dst.append(fresh[0])
                row[-1] = fresh[0]
                fresh = fresh[1:]
            row += fresh
            got.append(want[b])
        else:
            got.append(kept[b])
        out.append(row + [-1] * (C - len(row)))
    fill = [-1] * (S - len(src))
    return {"table": out, "lengths": kept, "room": got, "src": src + fill, "dst": dst + fill,
            "count": [len(src), len(free) - taken]}


def compact(table, lengths, pages, P):
    """include/rrs.h, rrs_kv_compact: a dict of lists."""
    C = len(table[0])
    rows = [row[:-(-min(max(n, 0), C * P) // P)] for row, n in zip(table, lengths)]
    used = sorted({p for row in rows for p in row if 0 <= p < pages})
    holes = [p for p in range(len(used)) if p not in set(used)]
    moves = [p for p in used if p >= len(used)]
    assert len(holes) == len(moves)
    to = dict(zip(moves, holes))
    out = [[to.get(p, p) for p in row] + [-1] * (C - len(row)) for row in rows]
    fill = [-1] * (max(1, pages // 2) - len(moves))
    return {"table": out, "src": moves + fill, "dst": holes + fill,
            "count": [len(moves), len(used)]}
