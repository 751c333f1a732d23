"""Oracle: a paged cache of K and V, and attention over it, in fp64 and integers (test infrastructure).

Row j of sequence b, rows row_start[b] .. row_start[b+1] - 1 of the dense tensors, has position kv_len[b] - n_b + j; position t lies in
slot t % page_size of page page_table[b][t // page_size].  An entry outside [0, n_pages) names no page: nothing is written there, rows
read from there are 0, its keys are not visible.  row_start counts as at least 0 and at most the number of rows.

e4m3 rows have one factor 2^e: the smallest e >= -100 with max|finite x| <= 448 * 2^e.
"""
import math

import numpy as np


def round_e4m3(x):
    """Nearest 8-bit float with 4 exponent and 3 mantissa bits (bias 7, no infinities), ties to even; NaN stays NaN.  |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(x == 0, 1.0, np.abs(x)))), -6.0)
        step = np.exp2(np.where(np.isfinite(e), e, 0.0) - 3.0)
        return np.where(np.isnan(x), np.nan, np.round(x / step) * step)


def quantise(x):
    """x [..., d] -> (values [..., d], exponents [...]): x is about values * 2^exponents."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isfinite(x), x, np.nan)
    top = np.nanmax(np.where(np.isnan(x), 0.0, np.abs(x)), axis=-1)
    exps = np.empty(top.shape, dtype=np.int64)
    for i, t in np.ndenumerate(top):
        e = -100
        while t > math.ldexp(448.0, e):
            e += 1
        exps[i] = e
    limit = 1.875 * 2.0 ** 127
    x = np.clip(x, -limit, limit)
    return round_e4m3(x * np.exp2(-exps.astype(np.float64))[..., None]), exps


def clipped(row_start, n_rows):
    """row_start as it counts for tensors of n_rows rows."""
    return [min(max(int(x), 0), n_rows) for x in row_start]


def places(page_table, kv_len, row_start, page_size, n_pages, n_rows=None):
    """[(row, page, slot)] of all rows; page None where there is none.  n_rows: rows of the dense tensors (by default the list's last entry)."""
    got = []
    row_start = clipped(row_start, row_start[-1] if n_rows is None else n_rows)
    for b, kv in enumerate(kv_len):
        for row in range(row_start[b], row_start[b + 1]):
            pos = kv - row_start[b + 1] + row
            page = None
            if 0 <= pos < len(page_table[b]) * page_size and 0 <= page_table[b][pos // page_size] < n_pages:
                page = page_table[b][pos // page_size]
            got.append((row, page, pos % page_size))
    return got


def visible(pos, kv, causal, window, sinks):
    """Positions that the row at `pos` of a sequence of kv tokens sees."""
    t = np.arange(kv)
    if not causal:
        return t
    ok = t <= pos
    if window > 0:
        ok &= (t > pos - window) | (t < sinks)
    return t[ok]


def attention(q, k_pages, v_pages, page_table, kv_len, row_start, causal=True, window=0, sinks=0, scale=None):
    """q [rows, Hq, d]; k_pages, v_pages [n_pages, Hkv, page_size, d] (the values the cache stands for).
    Returns (out [rows, Hq, d], lse [rows, Hq], size): rows of no sequence are NaN; size [rows, Hq, d] holds sum p |v|, the scale of
    rounding errors of the probabilities, and its companion reach [rows, Hq] the largest sum |q k| scale of a visible key."""
    q, k_pages, v_pages = (np.asarray(x, dtype=np.float64) for x in (q, k_pages, v_pages))
    rows, hq, d = q.shape
    n_pages, hkv, ps, _ = k_pages.shape
    row_start = clipped(row_start, rows)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, size = np.full((rows, hq, d), np.nan), np.full((rows, hq, d), np.nan)
    lse, reach = np.full((rows, hq), np.nan), np.zeros((rows, hq))
    for b, kv in enumerate(kv_len):
        table = np.asarray(page_table[b])
        n = row_start[b + 1] - row_start[b]
        for j in range(n):
            t = visible(kv - n + j, kv, causal, window, sinks)
            t = t[t < len(table) * ps]
            pages = table[t // ps] if len(t) else np.zeros(0, dtype=np.int64)
            t = t[(pages >= 0) & (pages < n_pages)]
            row = row_start[b] + j
            if not len(t):
                out[row], size[row], lse[row] = 0.0, 0.0, -np.inf
                continue
            k, v = k_pages[table[t // ps], :, t % ps], v_pages[table[t // ps], :, t % ps]         # [keys, hkv, d]
            for h in range(hq):
                g = h * hkv // hq
                with np.errstate(all="ignore"):
                    s = k[:, g] @ q[row, h] * scale
                    m = s.max()
                    p = np.exp(s - m)
                    lse[row, h] = m + np.log(p.sum())
                    p /= p.sum()
                    out[row, h] = p @ v[:, g]
                    size[row, h] = p @ np.abs(v[:, g])
                    reach[row, h] = (np.abs(k[:, g]) @ np.abs(q[row, h])).max() * scale
    return out, lse, size, reach
