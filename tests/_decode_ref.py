"""Plain float64 statements of the decode-side operators, and inputs for their tests.  Host only (numpy)."""
import numpy as np

EPS_BF16 = 2.0 ** -8          # a rounding to bf16: half a step, relative


def bf16_values(rng, *shape, scale=1.0):
    """Normal values that bf16 holds exactly (float64 array)."""
    x = (rng.standard_normal(shape) * scale).astype(np.float32)
    return ((x.view(np.uint32) + 0x8000) & 0xFFFF0000).view(np.float32).astype(np.float64)


def page_tables(past, new, page, free, table, rows, parents=None, words=0):
    """(table, seq_lens, row_start, positions, slots, bits, info) with None where nothing is written."""
    table = np.array(table)
    n, width = table.shape
    positions, slots = [None] * rows, [None] * rows
    bits = [None] * rows
    start, taken, failed, row_start = 0, 0, 0, [0]
    for b in range(n):
        p, f = max(past[b], 0), max(new[b], 0)
        bad = past[b] < 0 or new[b] < 0 or p + f > width * page or (parents is not None and f > 32 * words)
        held = -(-min(p, width * page) // page)
        upto = -(-min(p + f, width * page) // page)
        for c in range(held, upto):
            if taken < len(free):
                table[b, c] = free[taken]
            else:
                table[b, c] = -1
                bad = True
            taken += 1
        for j in range(f):
            t = start + j
            if t >= rows:
                break
            c = (p + j) // page
            slots[t] = -1 if c >= width or table[b, c] < 0 else int(table[b, c]) * page + (p + j) % page
            depth = j
            if parents is not None:
                seen, x = [], j
                while x >= 0:
                    seen.append(x)
                    up = parents[start + x]
                    x = up if -1 <= up < x else -1
                depth = len(seen) - 1
                bits[t] = [sum(1 << (x % 32) for x in seen if x // 32 == w) for w in range(words)]
            positions[t] = p + depth
        start += f
        failed += bad
        row_start.append(start)
    lens = [max(p, 0) + max(f, 0) for p, f in zip(past, new)]
    return table, lens, row_start, positions, slots, bits, [start, min(taken, len(free)), failed, max(lens)]


def norm_rope(x, weight, eps, inv_freq, interleaved, positions):
    """x [heads, rows, d] -> (result, bound of the fp32 arithmetic's error)."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    n = len(inv_freq)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq)
    c, s = np.cos(angle), np.sin(angle)
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    a, b = x[..., ia], x[..., ib]
    y, size = x.copy(), np.abs(x)
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = np.abs(a) + np.abs(b)
    # fp32: the mean of 128 squares, the root and the products are off by under 2^-19 relative, the angle's sine and
    # cosine by under 2^-21 of a turn's unit circle
    return y, size * 2.0 ** -18


def visible(n, past, bits_rows=None):
    """[n, past + n] truth values."""
    seen = np.ones((n, past + n), dtype=bool)
    for j in range(n):
        for x in range(n):
            seen[j, past + x] = x <= j if bits_rows is None else x // 32 < len(bits_rows[j]) and bool((bits_rows[j][x // 32] >> (x % 32)) & 1)
    return seen


def attention(q, k, v, seen):
    """One head of one request: q [n, d], k, v [len, d], seen [n, len] -> out, lse, bound of out's error, all float64.
    Masked keys take no part whatever they hold; a logit of -infinity weighs nothing, as a mask would."""
    n, d = q.shape
    out, lse, tol = np.zeros((n, d)), np.full(n, -np.inf), np.zeros((n, d))
    for j in range(n):
        idx = np.nonzero(seen[j])[0]
        z = k[idx] @ q[j] / np.sqrt(d)
        idx, z = idx[~np.isneginf(z)], z[~np.isneginf(z)]
        if len(idx) == 0:
            continue
        top = z.max()
        p = np.exp(z - top)
        total = p.sum()
        lse[j] = top + np.log(total)
        p = p / total
        out[j] = p @ v[idx]
        # one rounding of the result; each probability rounded to bf16 once; logits off by at most d 2^-24 sum|q k| / sqrt(d),
        # which stays below 2^-12 for the tests' inputs (d = 128, |q| |k| / sqrt(d) < 32)
        tol[j] = EPS_BF16 * np.abs(out[j]) + (EPS_BF16 + 2.0 ** -11) * (p @ np.abs(v[idx]))
    return out, lse, tol
