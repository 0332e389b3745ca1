"""Oracle of the packed-batch operators (include/vf.h, "packed batches over the page pool"): pages for the tokens
of a step, rotary embedding, attention of packed rows.  numpy, float64, written as the definitions read."""
import numpy as np

PAGE = 64


def _pages(tokens):
    return -(-tokens // PAGE)


def pages_assign(lens, new, free_pages, n_free, table, total_rows):
    """Returns (table, row_off, pos, slot, kv_len, n_free) after the step."""
    table, n = np.array(table, dtype=np.int32), len(lens)
    free, width = [int(p) for p in free_pages[:max(0, min(n_free, len(free_pages)))]], table.shape[1]
    had, wanted, row = len(free), 0, 0
    row_off, kv_len = np.zeros(n + 1, np.int32), np.zeros(n, np.int32)
    pos, slot = np.full(total_rows, -1, np.int32), np.full(total_rows, -1, np.int32)
    for b in range(n):
        h, w = int(lens[b]), int(new[b])
        ok = h >= 0 and w >= 0 and h + w <= PAGE * width
        need = _pages(h + w) - _pages(h) if ok else 0
        wanted += need
        ok = ok and (need == 0 or wanted <= had)
        if ok:
            for j in range(need):
                table[b, _pages(h) + j] = free.pop()
            kv_len[b] = h + w
        for j in range(min(max(w, 0), total_rows - row)):
            if ok:
                page = int(table[b, (h + j) // PAGE])
                pos[row + j] = h + j
                slot[row + j] = PAGE * page + (h + j) % PAGE if page >= 0 else -1
        row = min(row + max(w, 0), total_rows)
        row_off[b + 1] = row
    return table, row_off, pos, slot, kv_len, len(free)


def rotary_table(rotary_dim, theta, positions, scaling="unscaled", factor=1.0, low=0.0, high=0.0, trained=0.0, magnitude=1.0):
    i = np.arange(rotary_dim // 2)
    if scaling == "base":
        theta = theta * factor ** (rotary_dim / (rotary_dim - 2))
    f = theta ** (-2.0 * i / rotary_dim)
    if scaling == "positions":
        f = f / factor
    if scaling == "ramp":
        turns = trained * f / (2 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0, 1)
        f = f * keep + f / factor * (1 - keep)
    a = np.arange(positions)[:, None] * f
    return magnitude * np.stack([np.cos(a), np.sin(a)], -1)


def rotate(x, angles, interleaved):
    """x [rows, heads, hd], angles [rows, rotary_dim / 2, 2]."""
    x, y, half = np.asarray(x, np.float64), np.array(x, np.float64), angles.shape[1]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = angles[:, i, 0:1], angles[:, i, 1:2]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def pool_place(hd):
    """(offset of K[key][d], offset of V[key][d]) inside a page's block of one head, [64, hd] each."""
    k, v = np.zeros((PAGE, hd), np.int64), np.zeros((PAGE, hd), np.int64)
    for key in range(PAGE):
        tile, u, h, r = key // 32, key % 32 // 8, key % 8 // 4, key % 4
        for d in range(hd):
            k[key, d] = np.ravel_multi_index((tile, h, d // 32, d % 32 // 8, u, r, d % 8), (2, 2, hd // 32, 4, 4, 4, 8))
            v[key, d] = np.ravel_multi_index((tile, d // 16, key % 32 // 8, d % 16, key % 8), (2, hd // 16, 4, 16, 8))
    return k, v


def attention_packed(q, keys, values, row_off, kv_len, scale=None, present=None):
    """q [rows, q heads, hd]; keys, values: per sequence [tokens, kv heads, hd]; present: per sequence a truth value per token
    (False: its page is not there).  Returns (out, sum of |weight * value|: what rounding errors are measured against,
    largest sum of |q_i k_i| * scale of a score that counts); rows outside the offsets stay zero."""
    rows, hq, hd = q.shape
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    out, spread, size = np.zeros((rows, hq, hd)), np.zeros((rows, hq, hd)), np.zeros((rows, hq, 1))
    for b, n in enumerate(kv_len):
        r0, r1 = row_off[b], row_off[b + 1]
        k, v = np.asarray(keys[b][:n], np.float64), np.asarray(values[b][:n], np.float64)
        group = hq // k.shape[1]
        for r in range(r0, r1):
            seen = np.arange(n) <= n - (r1 - r0) + (r - r0)
            if present is not None:
                seen &= np.asarray(present[b][:n])
            if not seen.any():
                continue
            for h in range(hq):
                ks, vs, qs = k[seen, h // group], v[seen, h // group], np.asarray(q[r, h], np.float64)
                s = scale * (ks @ qs)
                w = np.exp(s - s.max())
                w /= w.sum()
                out[r, h], spread[r, h] = w @ vs, w @ np.abs(vs)
                size[r, h] = scale * (np.abs(ks) @ np.abs(qs)).max()
    return out, spread, size
