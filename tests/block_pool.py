"""A plain model of a paged cache's block tables, row by row: what gr_block_plan is compared with."""

OK, NO_BLOCKS, ROW_FULL, BAD_ROW = 0, 8, 9, 10


def plan(table, lengths, refs, block, beams, append, max_tokens, keep=None, parents=None):
    """Changes table (a list of lists), lengths and refs (lists) and returns slots, positions, offsets, copy_src,
    copy_dst, status."""
    R, N = len(lengths), len(refs)
    width = len(table[0]) if R else 0
    most = width * block
    old = [list(r) for r in table]
    old_len = list(lengths)
    div_up = lambda a: -(-a // block)
    base, kept, ask, status, offsets, end = [], [], [], [], [0], 0
    for r in range(R):
        st = BAD_ROW if append[r] < 0 else OK
        p = r
        if parents is not None:
            p = r // beams * beams + parents[r] if 0 <= parents[r] < beams else None
            if not -1 <= parents[r] < beams:
                st = BAD_ROW
        n = 0 if p is None else old_len[p]
        if not 0 <= n <= most:
            st, n = BAD_ROW, min(max(n, 0), most)
        if keep is not None:
            n = min(n, max(0, keep[r]))
        before = div_up(min(max(old_len[r], 0), most))
        now = [] if p is None else old[p][:div_up(n)]
        if any(not 0 <= b < N for b in now):
            bad_id = True
        else:
            bad_id = False
        for b in old[r][:before]:
            if 0 <= b < N:
                refs[b] -= 1
        for b in now:
            if 0 <= b < N:
                refs[b] += 1
        for c in range(before):
            table[r][c] = -1
        table[r][:len(now)] = now
        a = max(0, append[r])
        end += a
        if st == OK and (n + a > most or end > max_tokens):
            st = ROW_FULL
        if bad_id:
            st = BAD_ROW if st in (OK, ROW_FULL) else st
        base.append(n); kept.append(len(now)); ask.append(a if st == OK else 0); status.append(st)
        offsets.append(min(end, max_tokens))
    # who writes to a partly filled block
    writers = {}
    for r in range(R):
        if ask[r] and base[r] % block:
            writers.setdefault(table[r][base[r] // block], []).append(r)
    copies = [False] * R
    for b, rows in writers.items():
        if refs[b] > 1:
            stay = None
            if len(rows) == refs[b]:
                stay = min(rows, key=lambda r: (-(base[r] % block), r))
            for r in rows:
                copies[r] = r != stay
    free = [i for i in range(N) if refs[i] == 0]
    upto = 0
    src, dst = [-1] * R, [-1] * R
    for r in range(R):
        if status[r] != OK:
            continue
        need = int(copies[r]) + div_up(base[r] + ask[r]) - kept[r]
        start = upto
        upto += need
        if need and upto > len(free):
            status[r], ask[r] = NO_BLOCKS, 0
            continue
        mine = free[start:upto]
        if copies[r]:
            c = base[r] // block
            src[r], dst[r] = table[r][c], mine.pop(0)
            refs[src[r]] -= 1
            refs[dst[r]] += 1
            table[r][c] = dst[r]
        for i, b in enumerate(mine):
            table[r][kept[r] + i] = b
            refs[b] += 1
    slots, positions = [-1] * max_tokens, [-1] * max_tokens
    at = 0
    for r in range(R):
        lengths[r] = base[r] + ask[r]
        for k in range(ask[r]):
            t = base[r] + k
            slots[at + k] = table[r][t // block] * block + t % block
            positions[at + k] = t
        at += max(0, append[r])
    return slots, positions, offsets, src, dst, status
