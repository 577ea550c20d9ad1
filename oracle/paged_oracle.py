"""Plain float64 implementations of the paged cache's calls (test infrastructure): pages and slots, rows into slots, page scores and
selection, attention of one new token.  Written from the definitions in include/pact.h with loops over requests and rows."""
import numpy as np

OK, INVALID, NO_PAGES = 0, -1, -6


def pages_for(rows, page):
    return -(-rows // page)


def plan(page, table, length, n_new, free_pages, n_free, n_rows, row_stride=0):
    """Returns (status, table, length, free stack as a list up to its top, row_start, slot)."""
    B, width = table.shape
    table, lens = table.copy(), [int(x) for x in length]
    stack = [int(x) for x in free_pages[:max(0, int(n_free))]]
    nothing = (table.copy(), list(lens), list(stack), [0] * (B + 1), [-1] * n_rows)
    if not 0 <= n_free <= len(free_pages):
        return (INVALID,) + nothing
    rows = [max(0, int(m)) for m in n_new]
    for b in range(B):
        if lens[b] < 0 or lens[b] + rows[b] > width * page or (row_stride and rows[b] > row_stride):
            return (INVALID,) + nothing
    if sum(rows) > n_rows:
        return (INVALID,) + nothing
    for b in range(B):
        if n_new[b] < 0:
            stack += [int(x) for x in table[b, :pages_for(lens[b], page)]]
            lens[b] = 0
    if len(stack) > len(free_pages):
        return (INVALID,) + nothing
    if sum(pages_for(lens[b] + rows[b], page) - pages_for(lens[b], page) for b in range(B)) > len(stack):
        return (NO_PAGES,) + nothing
    start, slot = [0], [-1] * n_rows
    for b in range(B):
        for place in range(pages_for(lens[b], page), pages_for(lens[b] + rows[b], page)):
            table[b, place] = stack.pop()
        for i in range(rows[b]):
            p = lens[b] + i
            slot[(b * row_stride if row_stride else start[b]) + i] = int(table[b, p // page]) * page + p % page
        lens[b] += rows[b]
        start.append(start[b] + rows[b])
    return OK, table, lens, stack, start, slot


def write(K, V, logw, bounds, w_max, K_new, V_new, logw_new, slot, page):
    """In place on [n_pages, n_kvh, page, d_h] arrays and the like; returns the status."""
    status, n_pages = OK, K.shape[0]
    for r, s in enumerate(slot):
        if s < 0:
            continue
        if s >= n_pages * page:
            status = INVALID
            continue
        at, place = divmod(int(s), page)
        K[at, :, place], V[at, :, place] = K_new[r], V_new[r]
        w = 0.0 if logw_new is None or logw is None else logw_new[r]
        if logw is not None:
            logw[at, place] = w
        if bounds is not None:
            if place == 0:
                bounds[at, :, 0], bounds[at, :, 1], w_max[at] = K_new[r], K_new[r], w
            else:
                bounds[at, :, 0] = np.fmin(bounds[at, :, 0], K_new[r])
                bounds[at, :, 1] = np.fmax(bounds[at, :, 1], K_new[r])
                w_max[at] = np.fmax(w_max[at], w)
    return status


def page_scores(q, bounds, w_max, ids, scale):
    """q [g, d_h] of one key head, bounds [n_pages, 2, d_h] of it -> the score of each page of ids."""
    out = []
    for at in ids:
        if not 0 <= at < len(bounds):
            out.append(-np.inf)
            continue
        with np.errstate(invalid="ignore"):                # (infinities: 0 times one is no part of the sum, two of them may make a NaN)
            s = (np.where(q == 0, 0.0, q * np.where(q > 0, bounds[at, 1], bounds[at, 0]))).sum(1) * scale
        s = s[~np.isnan(s)]
        with np.errstate(invalid="ignore"):
            s = max(s) + w_max[at] if len(s) else -np.inf
        out.append(-np.inf if np.isnan(s) else s)
    return np.array(out)


def select(q, bounds, w_max, table, length, page, scale, n_first, n_last, n_select):
    """q [B, n_qh, d_h], bounds [n_pages, n_kvh, 2, d_h] -> [B, n_kvh, n_select]."""
    B, n_qh, _ = q.shape
    H = bounds.shape[1]
    g = n_qh // H
    out = np.full((B, H, n_select), -1, np.int32)
    for b in range(B):
        n = pages_for(min(max(int(length[b]), 0), table.shape[1] * page), page)
        for h in range(H):
            if n <= n_select:
                out[b, h, :n] = np.arange(n)
                continue
            s = page_scores(q[b, h * g:(h + 1) * g], bounds[:, h], w_max, table[b, :n], scale)
            forced = list(range(n_first)) + list(range(n - n_last, n))
            rest = sorted(range(n_first, n - n_last), key=lambda p: (-s[p], p))
            out[b, h] = sorted(forced + rest[:n_select - len(forced)])
    return out


def rows_of(table, length, page, n_pages, selected=None):
    """(page id, place) of the rows that one request's token attends to, in order; selected: places of one key head."""
    n = pages_for(length, page)
    places = range(n) if selected is None else list(selected[:min(len(selected), n)])
    out = []
    for place in places:
        if 0 <= place < n and 0 <= table[place] < n_pages:
            out += [(int(table[place]), r) for r in range(min(page, length - place * page))]
    return out


def attend(q, K, V, logw, table, length, page, scale, selected=None):
    """Returns out [B, n_qh, d_h], lse [B, n_qh], and what a tolerance needs: sum_p w_p |v_p| per element and the largest
    scale * sum_c |q_c k_pc| + |logw_p| per head."""
    B, n_qh, D = q.shape
    H = K.shape[1]
    g = n_qh // H
    out, mag = np.zeros((B, n_qh, D)), np.zeros((B, n_qh, D))
    lse, big = np.full((B, n_qh), -np.inf), np.zeros((B, n_qh))
    for b in range(B):
        n = min(max(int(length[b]), 0), table.shape[1] * page)
        for h in range(H):
            rows = rows_of(table[b], n, page, K.shape[0], None if selected is None else selected[b, h])
            if logw is not None:
                rows = [x for x in rows if logw[x] != -np.inf]
            if not rows:
                continue
            at = tuple(np.array(rows).T)
            k, v = K[at[0], h, at[1]], V[at[0], h, at[1]]
            w = 0.0 if logw is None else logw[at]
            for j in range(h * g, (h + 1) * g):
                s = k @ q[b, j] * scale + w
                m = s.max()
                e = np.exp(s - m)
                p = e / e.sum()
                out[b, j], mag[b, j] = p @ v, p @ np.abs(v)
                lse[b, j] = m + np.log(e.sum())
                big[b, j] = (np.abs(k) @ np.abs(q[b, j]) * abs(scale) + np.abs(w)).max()
    return out, lse, mag, big
