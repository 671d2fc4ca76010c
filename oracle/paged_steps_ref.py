"""Plain CPU statements of the decode steps over the paged cache of bf16 or fp32 rows: pages' bounds and their update, the choice of pages,
attention over a list of rows.  float64 and Python integers, written from the definitions; test infrastructure only."""
import math

import numpy as np


def bounds_of(rows):
    """Lowest and largest of each column of rows [n, d], NaNs left out."""
    low = np.where(np.isnan(rows), np.inf, rows).min(0)
    high = np.where(np.isnan(rows), -np.inf, rows).max(0)
    return low, high


def page_bounds(K, rows, table, page_size, bounds):
    """A copy of bounds [num_pages, 2, d] with those of the pages that hold rows."""
    out = bounds.copy()
    B, L, H, most = table.shape
    for b in range(B):
        for l in range(L):
            n = max(0, int(rows[b, l]))
            for h in range(H):
                for i in range(min(most, -(-n // page_size))):
                    page = int(table[b, l, h, i])
                    if 0 <= page < K.shape[0]:
                        out[page] = bounds_of(K[page, :min(page_size, n - i * page_size)])
    return out


def append_bounds(bounds, K_pages, slots, page_size):
    """bounds after rows went to the slots [B, H, T] of K_pages (their present contents)."""
    out = bounds.copy()
    B, H, T = slots.shape
    for b in range(B):
        for h in range(H):
            pages = {}
            for s in slots[b, h]:
                if 0 <= s < K_pages.shape[0] * page_size:
                    pages.setdefault(int(s) // page_size, []).append(int(s) % page_size)
            for page, places in pages.items():
                low, high = bounds_of(K_pages[page, places])
                if 0 not in places:
                    low, high = np.fmin(low, out[page, 0]), np.fmax(high, out[page, 1])
                out[page] = low, high
    return out


def page_score(q, low, high):
    """sum_g sum_c of the largest product of q_gc and a key from low_c to high_c, rounded to float32, of q [G, d]: q_gc high_c, of a negative query
    q_gc low_c, where 0 times infinity is 0.  Columns without numbers (+infinity, -infinity) reach from -infinity to +infinity."""
    none = (low == np.inf) & (high == -np.inf)
    bound = np.where(q < 0, np.where(none, -np.inf, low), np.where(none, np.inf, high))
    with np.errstate(invalid="ignore"):
        product = q * bound
        return float(np.float32(np.where(np.isnan(product) & ~np.isnan(q) & ~np.isnan(bound), 0.0, product).sum()))


def choose_pages(Q, bounds, rows, table, page_size, count, first, last):
    """Q float64 [B, L, Hq, d], bounds float64 [num_pages, 2, d]: places [B, L, H, count]."""
    B, L, H, most = table.shape
    G = Q.shape[2] // H
    out = np.full((B, L, H, count), -1, np.int32)
    for b in range(B):
        for l in range(L):
            blocks = min(most, -(-max(0, int(rows[b, l])) // page_size))
            for h in range(H):
                q = Q[b, l, h * G:(h + 1) * G]
                ranked = []
                for i in range(blocks):
                    page = int(table[b, l, h, i])
                    if not 0 <= page < bounds.shape[0]:
                        continue
                    score = page_score(q, bounds[page, 0], bounds[page, 1])
                    forced = i < first or i >= blocks - last
                    ranked.append((0 if forced else 2 if math.isnan(score) else 1, 0.0 if forced or math.isnan(score) else -score, i))
                taken = sorted(i for _, _, i in sorted(ranked)[:count])
                out[b, l, h, :len(taken)] = taken
    return out


def rows_at(K, V, rows, table, page_size, places):
    """The rows of one unit (rows held, its table) in the pages at `places`, in order."""
    slots = []
    for i in places:
        if 0 <= i < len(table) and 0 <= table[i] < K.shape[0]:
            slots += [(int(table[i]), r) for r in range(max(0, min(page_size, int(rows) - int(i) * page_size)))]
    if not slots:
        return np.zeros((0, K.shape[2])), np.zeros((0, K.shape[2]))
    p, r = np.array(slots).T
    return K[p, r], V[p, r]


def attend(q, K, V, scale):
    """q [G, d], K and V [n, d] in float64: (result, sum p |v|, largest |logit|, largest sum |q k| |scale|)."""
    if not K.shape[0]:
        return np.zeros_like(q), np.zeros_like(q), 0.0, 0.0
    logit = q @ K.T * scale
    p = np.exp(logit - logit.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return p @ V, p @ np.abs(V), float(np.abs(logit).max()), float((np.abs(q) @ np.abs(K).T).max() * abs(scale))
