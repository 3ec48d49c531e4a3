"""Tables from lengths, block copies and attention with shared prefixes, from their definitions on the host: sequence by sequence and
block by block.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

import cache_reference as ref

OK, INVALID_ARG, NO_FREE_BLOCKS, BAD_BLOCK_ID = 0, 1, 4, 5
MOST = 1 << 30


def advance(T, table, refs, old, new, parents=None, shared=None, num_rows=None, first_pos=None, pairs_cap=0):
    """The step as it is documented.  num_rows None: rows are not numbered.  Returns a dict of what comes out; inputs keep."""
    table, refs, was, count = table.copy(), refs.copy(), table, refs
    S, width, NB = len(old), table.shape[1], len(refs)
    room = min(width * T, MOST)
    free = [int(b) for b in np.flatnonzero(refs == 0)]
    codes, lens = set(), [int(x) for x in old]
    taken = rows = 0
    pairs, starts, positions, slots = [], [0], [], []
    full = None  # why the growing sequences behind some one stay as they are
    plans = []
    good = lambda b: 0 <= b < NB  # noqa: E731
    for s in range(S):
        o, n = int(old[s]), int(new[s])
        t = -1 if parents is None else int(parents[s])
        ok = 0 <= o <= room and 0 <= n <= room and t < S
        if ok and t >= 0:
            sh = int(shared[s])
            ok = o == 0 and 0 <= sh <= int(old[t]) <= room and sh <= n
        if not ok:
            codes.add(INVALID_ARG)
            starts.append(rows)
            continue
        at = int(shared[s]) if t >= 0 else o
        grows = t >= 0 or n > o
        copy = False
        if at % T and grows:
            if t >= 0:
                copy = True
            else:
                b = int(was[s, at // T])
                if not good(b) or count[b] < 1:
                    codes.add(BAD_BLOCK_ID)
                else:
                    copy = count[b] > 1
        have = at // T if copy else -(-at // T)
        need = max(-(-n // T) - have, 0) if grows else 0
        fresh = n - at if grows and num_rows is not None else 0
        if grows and full is None:
            if taken + need > len(free):
                full = NO_FREE_BLOCKS
            elif (num_rows is not None and rows + fresh > num_rows) or len(pairs) + copy > pairs_cap:
                full = INVALID_ARG
            if full is not None:
                codes.add(full)
        if grows and full is not None:
            starts.append(rows)
            continue
        plans.append((s, t, at, copy, have, need, fresh, o, n))
        taken += need
        rows += fresh
        if copy:
            pairs.append(None)
        starts.append(rows)
    taken = k = 0
    for s, t, at, copy, have, need, fresh, o, n in plans:
        lens[s] = n
        if t >= 0:
            for j in range(at // T):
                b = int(was[t, j])
                table[s, j] = b
                if good(b) and count[b] > 0:
                    refs[b] += 1
                else:
                    codes.add(BAD_BLOCK_ID)
        if n < o:
            for j in range(-(-n // T), -(-o // T)):
                b = int(was[s, j])
                table[s, j] = -1
                if good(b) and count[b] > 0 and refs[b] > 0:
                    refs[b] -= 1
                else:
                    codes.add(BAD_BLOCK_ID)
        if copy:
            b = int(was[t if t >= 0 else s, at // T])
            known = good(b) and count[b] > 0
            pairs[k] = (b if known else -1, free[taken])
            k += 1
            if not known:
                codes.add(BAD_BLOCK_ID)
            elif t < 0:
                refs[b] -= 1
        for j in range(need):
            table[s, have + j] = free[taken]
            refs[free[taken]] = 1
            taken += 1
        for j in range(fresh):
            i = at + j
            positions.append(i if first_pos is None else int(first_pos[s]) + j)
            b = int(table[s, i // T])
            slots.append(b * T + i % T if good(b) else -1)
    out = dict(table=table, refs=refs, lens=np.array(lens, np.int32), pairs=np.array(pairs, np.int32).reshape(-1, 2),
               free=int((refs == 0).sum()), status=next((c for c in (INVALID_ARG, NO_FREE_BLOCKS, BAD_BLOCK_ID) if c in codes), OK))
    if num_rows is not None:
        pad = num_rows - len(slots)
        out.update(starts=np.array(starts, np.int32), positions=np.array(positions + [0] * pad, np.int32),
                   slots=np.array(slots + [-1] * pad, np.int64))
    return out


def tolerance_shared(dtype, D, n, out, absv, size, vmax):
    """As for attention by itself, and for the join of the two sums: two exponentials of 2^-21 each beside the largest, and a product
    and an addition of half a step of 2^-23 in the numerator and in the sum."""
    join = 2 * (2.0 ** -20 + 2 * 2.0 ** -23)
    return ref.tolerance_attend(dtype, D, n, out, absv, size, vmax) + join * (absv + np.abs(out))


def tolerance_shared_lse(D, n, lse, size):
    return ref.tolerance_lse(D, n, lse, size) + 2.0 ** -19
