"""Fork and compact as a program on lists: one sequence after the other, from a sorted list of the free pages."""


def columns_of(rows, page_rows):
    return -(-rows // page_rows)


def fork(pages, lengths, holders, parents, wanted, page_rows, window=None, sinks=0):
    """Lists of lists and numbers.  Returns pages, lengths, holders and moves."""
    count, columns = len(holders), len(pages[0]) if pages else 0
    room = columns * page_rows
    holders = list(holders)
    is_page = lambda p: 0 <= p < count      # noqa: E731
    for row, n in zip(pages, lengths):
        if 0 <= n <= room:
            for p in row[:columns_of(n, page_rows)]:
                if is_page(p):
                    holders[p] -= 1
    plans, first = [], {}
    for i, parent in enumerate(parents):
        n = 0 if parent == -1 else lengths[parent] if 0 <= parent < len(lengths) else -1
        want = n if wanted is None else wanted[i]
        if not (-1 <= parent < len(lengths)) or not 0 <= n <= room or not 0 <= want <= room:
            plans.append(None)
            continue
        kept = min(n, want)
        row, part = [-1] * columns, -1
        for c in range(columns_of(kept, page_rows)):
            gone = window is not None and c * page_rows >= sinks and (c + 1) * page_rows <= kept - window
            if not gone and is_page(pages[parent][c]):
                row[c] = pages[parent][c]
        if kept % page_rows:
            part = row[kept // page_rows]
        for c, p in enumerate(row):
            if p >= 0 and not (part >= 0 and c == kept // page_rows):
                holders[p] += 1
        if part >= 0:
            first.setdefault(part, i)
        plans.append((kept, want, row, part))
    free = [p for p in range(count) if holders[p] == 0 and p not in first]
    whole = list(holders)     # holders of whole pages
    out, after, moves, taken = [], [], [], 0
    for i, plan in enumerate(plans):
        if plan is None:
            out.append([-1] * columns)
            after.append(-1)
            moves.append([-1, -1, 0])
            continue
        kept, want, row, part = plan
        copies = part >= 0 and not (first[part] == i and whole[part] == 0)
        need = copies + columns_of(want, page_rows) - columns_of(kept, page_rows)
        if need and taken + need > len(free):
            for c, p in enumerate(row):
                if p >= 0 and not (part >= 0 and c == kept // page_rows):
                    holders[p] -= 1
            taken += need
            out.append([-1] * columns)
            after.append(-1)
            moves.append([-1, -1, 0])
            continue
        take = free[taken:taken + need]
        taken += need
        move = [-1, -1, 0]
        if part >= 0:
            if copies:
                move = [part, take[0], kept % page_rows]
                row[kept // page_rows] = take[0]
            else:
                holders[part] = 1
        for c, p in zip(range(columns_of(kept, page_rows), columns), take[copies:]):
            row[c] = p
        for p in take:
            holders[p] = 1
        out.append(row)
        after.append(want)
        moves.append(move)
    return out, after, holders, moves


def compact(pages, lengths, holders, page_rows):
    """Returns pages, holders and moves."""
    count, columns = len(holders), len(pages[0]) if pages else 0
    used = sum(h != 0 for h in holders)
    high = [p for p in range(used, count) if holders[p]]
    low = [p for p in range(used) if not holders[p]]
    to = dict(zip(high, low))
    after = list(holders)
    for p, x in to.items():
        after[x], after[p] = holders[p], 0
    out = [[to.get(p, p) if 0 <= n <= columns * page_rows and c < columns_of(n, page_rows) else p for c, p in enumerate(row)] for row, n in zip(pages, lengths)]
    moves = [[p, x, page_rows] for p, x in to.items()]
    return out, after, moves + [[-1, -1, 0]] * (count // 2 - len(moves))
