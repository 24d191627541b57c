"""The page operations of a paged cache written out one request at a time on the host: what the library's calls do to the
page table, the reference counts and the pool (numpy arrays, changed in place). Each call returns the status bits."""
import numpy as np

BAD_PAGE, CTX_OVERFLOW, BAD_ROW, POOL_FULL = 2, 4, 16, 32


def _free(ref):
    return [p for p in range(len(ref)) if ref[p] <= 0]


def copy(pool, src, dst, n_slots=None, count=None):
    n = len(src) if count is None else max(0, min(len(src), int(count)))
    pages, ps = pool.shape[1], pool.shape[4]
    status, todo = 0, []
    for i in range(n):
        if src[i] < 0:
            continue
        bad = src[i] >= pages or not 0 <= dst[i] < pages
        bad |= any(src[k] >= 0 and (src[k] == dst[i] or (k < i and dst[k] == dst[i])) for k in range(n))
        if bad:
            status |= BAD_PAGE
            continue
        todo.append((src[i], dst[i], ps if n_slots is None else min(max(int(n_slots[i]), 0), ps)))
    old = pool.copy()
    for s, d, k in todo:
        pool[:, d, :, :, :k] = old[:, s, :, :, :k]
    return status


def fork(table, ref, pool, parent, child, fork_len):
    rows, width = table.shape
    pages, ps = pool.shape[1], pool.shape[4]
    old, status, free, n_free = table.copy(), 0, _free(ref), None
    n_free, used, copies = len(free), 0, []
    for i, (p, c, n) in enumerate(zip(parent, child, fork_len)):
        copies.append((-1, -1, 0))
        n = max(int(n), 0)
        need_pages = -(-n // ps)
        if not (0 <= p < rows and 0 <= c < rows) or p == c:
            status |= BAD_ROW
            continue
        if need_pages > width:
            status |= CTX_OVERFLOW
            continue
        bits = 0
        if p in child or c in child[:i] or (old[c] >= 0).any():
            bits |= BAD_ROW
        if ((old[p, :need_pages] < 0) | (old[p, :need_pages] >= pages)).any():
            bits |= BAD_PAGE
        status |= bits
        if bits:
            continue
        whole, rest = divmod(n, ps)
        if rest:
            used += 1
            if used > n_free:
                status |= POOL_FULL
                continue
        table[c] = -1
        for j in range(whole):
            table[c, j] = old[p, j]
            ref[old[p, j]] += 1
        if rest:
            page = free[used - 1]
            table[c, whole], ref[page] = page, 1
            pool[:, page, :, :, :rest] = pool[:, old[p, whole], :, :, :rest]
            copies[-1] = (int(old[p, whole]), page, rest)
    return status, copies


def resize(table, ref, pool, rows, keep_len, capacity):
    n_rows, width = table.shape
    pages, ps = pool.shape[1], pool.shape[4]
    old, old_ref, old_pool, status = table.copy(), ref.copy(), pool.copy(), 0
    free, used, copies, gained = _free(ref), 0, [], []
    for i, (r, n, cap) in enumerate(zip(rows, keep_len, capacity)):
        copies.append((-1, -1, 0))
        cap = max(int(cap), 0)
        n = min(max(int(n), 0), cap)
        want, first = -(-cap // ps), n // ps
        if not 0 <= r < n_rows:
            status |= BAD_ROW
            continue
        if want > width:
            status |= CTX_OVERFLOW
            continue
        bits = BAD_ROW if r in rows[:i] else 0
        e = old[r]
        if (e >= pages).any() or (e[:-(-n // ps)] < 0).any():
            bits |= BAD_PAGE
        status |= bits
        if bits:
            continue
        fresh = [j for j in range(want) if e[j] < 0 or (j >= first and n < cap and old_ref[e[j]] > 1)]
        if fresh:
            used += len(fresh)
            if used > len(free):
                status |= POOL_FULL
                continue
        base = used - len(fresh)
        for j in range(width):
            if e[j] >= 0 and (j >= want or j in fresh):
                ref[e[j]] -= 1
            if j in fresh:
                page = free[base + fresh.index(j)]
                table[r, j] = page
                gained.append(page)
                if j == first and n % ps and e[j] >= 0:
                    pool[:, page, :, :, :n % ps] = old_pool[:, e[j], :, :, :n % ps]
                    copies[-1] = (int(e[j]), page, n % ps)
            elif j >= want:
                table[r, j] = -1
    for page in gained:
        ref[page] = 1
    return status, copies


def compact(table, ref, pool):
    pages = len(ref)
    live = int((ref > 0).sum())
    holes = [p for p in range(live) if ref[p] <= 0]
    movers = [p for p in range(live, pages) if ref[p] > 0]
    to, status = dict(zip(movers, holes)), 0
    for s, d in to.items():
        pool[:, d] = pool[:, s]
        ref[d], ref[s] = ref[s], 0
    flat = table.reshape(-1)
    for i, e in enumerate(flat.copy()):
        if e >= live:
            if int(e) in to:
                flat[i] = to[int(e)]
            else:
                status |= BAD_PAGE
    return status, live, list(zip(movers, holes))
