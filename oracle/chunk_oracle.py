"""Plain float64 implementation of the attention of several new tokens per request over a paged cache, and of the calls for pages that several requests hold (test
infrastructure).  Written from the definitions in include/pact.h with loops over requests, heads and pages."""
import numpy as np

from .paged_oracle import INVALID, NO_PAGES, OK, pages_for


def attend(q, K, V, logw, table, length, n_new, start, page, scale, causal, n_rows, most=None):
    """q [n_rows, n_qh, d_h]; token i of request b is row start[b] + i, for at most `most` tokens.  Returns (touched [n_rows], out, lse, sum_p w_p |v_p| per element, largest
    scale * sum_c |q_c k_pc| + |logw_p| per head among the rows that count for more than nothing) as arrays over the rows."""
    n_qh, D = q.shape[1:]
    g = n_qh // K.shape[1]
    out, mag = np.zeros((n_rows, n_qh, D)), np.zeros((n_rows, n_qh, D))
    lse, big = np.full((n_rows, n_qh), -np.inf), np.zeros((n_rows, n_qh))
    touched = np.zeros(n_rows, bool)
    for b in range(len(length)):
        n, want, r0 = min(max(int(length[b]), 0), table.shape[1] * page), max(int(n_new[b]), 0), int(start[b])
        m = min(want, want if most is None else most, max(0, n_rows - r0)) if r0 >= 0 else 0
        touched[r0:r0 + m] = True
        # positions of the rows that are there (those of pages outside the cache are not)
        pos = np.array([p for p in range(n) if 0 <= table[b, p // page] < K.shape[0]], int)
        if m == 0 or len(pos) == 0:
            continue
        ids, places = table[b, pos // page], pos % page
        w = np.zeros(len(pos)) if logw is None else logw[ids, places]
        seen = (pos[None] <= n - want + np.arange(m)[:, None] if causal else np.ones((m, len(pos)), bool)) & (w != -np.inf)
        some = seen.any(1)
        for h in range(K.shape[1]):
            k, v = K[ids, h, places], V[ids, h, places]
            for j in range(h * g, (h + 1) * g):
                x = q[r0:r0 + m, j]
                s = np.where(seen, x @ k.T * scale + w, -np.inf)[some]
                top = s.max(1, keepdims=True)
                e = np.exp(s - top)
                p = e / e.sum(1, keepdims=True)
                at = r0 + np.flatnonzero(some)
                out[at, j], mag[at, j] = p @ v, p @ np.abs(v)
                lse[at, j] = top[:, 0] + np.log(e.sum(1))
                big[at, j] = np.where(e > 0, (np.abs(x) @ np.abs(k).T * abs(scale) + np.where(w == -np.inf, 0, np.abs(w)))[some], 0).max(1)
    return touched, out, lse, mag, big


def fork(page, table, length, source, rows, shared, free_pages, n_free):
    """Returns (status, table as lists of the pages of each request, lengths, shared, stack, copies)."""
    B, width = table.shape
    P = len(shared)
    lens, shared = [int(x) for x in length], [int(x) for x in shared]
    stack = [int(x) for x in free_pages[:max(0, min(int(n_free), P))]]
    old = [[int(p) for p in table[b, :pages_for(min(max(lens[b], 0), width * page), page)]] for b in range(B)]
    same = (old, lens, list(shared), list(stack), [])
    if not 0 <= n_free <= P or any(not 0 <= n <= width * page for n in lens) or any(not -1 <= s < B for s in source):
        return (INVALID,) + same
    want = [0 if s < 0 else lens[s] if rows is None else int(rows[b]) for b, s in enumerate(source)]
    if any(s >= 0 and not 0 <= want[b] <= lens[s] for b, s in enumerate(source)) or any(not 0 <= p < P for x in old for p in x):
        return (INVALID,) + same
    held = [0] * P
    for x in old:
        for p in x:
            held[p] += 1
    if any(held[p] and (shared[p] < 0 or shared[p] + 1 < held[p]) for p in range(P)):
        return (INVALID,) + same
    outside = [shared[p] + 1 - held[p] if held[p] else 0 for p in range(P)]
    whole = [old[s][:want[b] // page] if s >= 0 else [] for b, s in enumerate(source)]
    full = [0] * P
    for x in whole:
        for p in x:
            full[p] += 1
    tail = [old[s][want[b] // page] if s >= 0 and want[b] % page else None for b, s in enumerate(source)]
    keeper = {}
    for b, p in enumerate(tail):
        if p is not None and p not in keeper and not full[p] and not outside[p]:
            keeper[p] = b
    now = [outside[p] + full[p] + (p in keeper) for p in range(P)]
    seen, freed = set(), []
    for x in old:
        for p in x:
            if p not in seen:
                seen.add(p)
                if now[p] == 0:
                    freed.append(p)
    copying = [b for b, p in enumerate(tail) if p is not None and keeper.get(p) != b]
    if len(stack) + len(freed) > P:
        return (INVALID,) + same
    if len(copying) > len(stack) + len(freed):
        return (NO_PAGES,) + same
    stack += freed
    copies, new = [], [list(x) for x in whole]
    for b, p in enumerate(tail):
        if p is None:
            continue
        if keeper.get(p) == b:
            new[b].append(p)
        else:
            fresh = stack.pop()
            copies.append([p, fresh, want[b] % page])
            new[b].append(fresh)
    for p in seen:
        shared[p] = max(now[p] - 1, 0)
    return OK, new, want, shared, stack, copies


def compact(page, table, length, shared, free_pages, n_free):
    """Returns (status, table as lists, shared, stack, moved_to, moves)."""
    B, width = table.shape
    P = len(shared)
    status = OK
    lens = [min(max(int(n), 0), width * page) for n in length]
    if any(int(n) != m for n, m in zip(length, lens)):
        status = INVALID
    old = [[int(p) for p in table[b, :pages_for(lens[b], page)]] for b in range(B)]
    if any(not 0 <= p < P for x in old for p in x):
        status = INVALID
    fits = 0 <= n_free <= P
    stack = [int(p) for p in free_pages[:n_free]] if fits else []
    if not fits or len(set(stack)) != len(stack) or any(not 0 <= p < P for p in stack):
        return INVALID, old, [int(x) for x in shared], stack, list(range(P)), []
    n_used, is_free = P - n_free, set(stack)
    holes = [p for p in range(n_used) if p in is_free]
    strays = [p for p in range(n_used, P) if p not in is_free]
    moved, shared = list(range(P)), [int(x) for x in shared]
    for s, h in zip(strays, holes):
        moved[s] = h
        shared[h], shared[s] = shared[s], 0
    return status, [[moved[p] if 0 <= p < P else p for p in x] for x in old], shared, list(range(P - 1, n_used - 1, -1)), moved, [[s, h, page] for s, h in zip(strays, holes)]
