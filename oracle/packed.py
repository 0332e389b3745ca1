"""Oracle of the packed-batch operators (include/vf.h, "packed batches over the page pool" and what follows it): pages for the
tokens of a step, rotary embedding, attention of packed rows; norms of heads; forks, tokens that stay, compaction of pages;
adjusted logits.  numpy, float64, written as the definitions read."""
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


def norm_heads(x, gain, eps):
    """x [rows, heads, hd]; gain [hd], [heads, hd] or None."""
    x = np.asarray(x, np.float64)
    x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x if gain is None else x * np.asarray(gain, np.float64)


def _held(length, width):
    return min(max(int(length), 0), PAGE * width)


def pages_fork(src, dst, tokens, lens, free_pages, n_free, table, shares):
    """Returns (table, shares, kv_len, copies, n_free) after the forks."""
    table, shares, kv_len = np.array(table, dtype=np.int32), np.array(shares, dtype=np.int32), np.array(lens, dtype=np.int32)
    n, width, pool = len(lens), table.shape[1], len(shares)
    free = [int(p) for p in free_pages[:max(0, min(int(n_free), len(free_pages)))]]
    had, wanted, copies, named = len(free), 0, [], set()
    for s, d, want in zip(src, dst, tokens):
        first = d not in named
        named.add(d)
        if not (0 <= s < n and 0 <= d < n) or not first or lens[d] > 0:
            continue
        held = _held(lens[s], width)
        t = held if want < 0 or want > held else int(want)
        full, part = t // PAGE, t % PAGE
        needs = part > 0 and 0 <= table[s, full] < pool
        wanted += needs
        if needs and wanted > had:
            continue
        for i in range(full):
            table[d, i] = table[s, i]
            if 0 <= table[s, i] < pool:
                shares[table[s, i]] += 1
        if needs:
            copies.append((int(table[s, full]), free.pop()))
            table[d, full] = copies[-1][1]
        elif part:
            table[d, full] = table[s, full]
        kv_len[d] = t
    return table, shares, kv_len, copies, len(free)


def pages_keep(lens, keep, free_pages, n_free, table, shares):
    """Returns (table, shares, kv_len, copies, free list) after the cuts."""
    table, shares = np.array(table, dtype=np.int32), np.array(shares, dtype=np.int32)
    n, width, pool = len(lens), table.shape[1], len(shares)
    free, room = [int(p) for p in free_pages[:max(0, min(int(n_free), len(free_pages)))]], len(free_pages)
    held = [_held(h, width) for h in lens]
    kept = [h if w < 0 or w > h else int(w) for h, w in zip(held, keep)]
    dropped = {}                                                   # page: times, in the order of the first
    for b in range(n):
        for t in range(_pages(kept[b]), _pages(held[b])):
            if 0 <= table[b, t] < pool:
                dropped[int(table[b, t])] = dropped.get(int(table[b, t]), 0) + 1
            table[b, t] = -1
    for page, times in dropped.items():
        if times > shares[page]:                                   # nobody is left
            if len(free) < room:
                free.append(page)
            shares[page] = 0
        else:
            shares[page] -= times
    cut = {}                                                       # page: the sequences that are cut inside it
    for b in range(n):
        t = kept[b] // PAGE
        if kept[b] < held[b] and kept[b] % PAGE and 0 <= table[b, t] < pool:
            cut.setdefault(int(table[b, t]), []).append(b)
    for page, who in cut.items():
        if len(who) > shares[page]:
            who.pop()                                              # keeps the page
        shares[page] -= len(who)
    copies = []
    for b in range(n):
        t = kept[b] // PAGE
        page = int(table[b, t]) if t < width else -1
        if kept[b] < held[b] and b in cut.get(page, []):
            if free:
                copies.append((page, free.pop()))
                table[b, t] = copies[-1][1]
            else:
                table[b, t] = -1
                kept[b] = PAGE * t
    return table, shares, np.array(kept, np.int32), copies, free


def pages_compact(lens, table, shares, room):
    """Returns (table, shares, free list, where every page went, copies) for a pool of `room` pages."""
    table, pool = np.array(table, dtype=np.int32), len(shares)
    n, width = table.shape
    pages = sorted({int(table[b, t]) for b in range(n) for t in range(_pages(_held(lens[b], width))) if 0 <= table[b, t] < pool})
    moved, out = np.full(pool, -1, np.int32), np.full((n, width), -1, np.int32)
    new_shares = np.zeros(room, np.int32)
    for i, page in enumerate(pages[:room]):
        moved[page], new_shares[i] = i, shares[page]
    for b in range(n):
        for t in range(_pages(_held(lens[b], width))):
            if 0 <= table[b, t] < pool:
                out[b, t] = moved[table[b, t]]
    return out, new_shares, list(range(len(pages), room)), moved, [(p, i) for i, p in enumerate(pages[:room])]


def logits_adjust(logits, row_off, penalties=None, history=None, prompt_len=None, tokens=None, biases=None, mask=None, mask_row=None):
    """logits [rows, vocab]; history: a list of ids per sequence; biases: per sequence a list of (id, value); mask [any, vocab] of
    truth values.  Rows outside the offsets come back as NaN."""
    z = np.asarray(logits, np.float64)
    rows, vocab = z.shape
    out = np.full(z.shape, np.nan)
    for b in range(len(row_off) - 1):
        for r in range(row_off[b], row_off[b + 1]):
            y = z[r].copy()
            if penalties is not None:
                rho, alpha, beta = (float(p) for p in penalties[b])
                text = [int(t) for t in history[b]] if history is not None else []
                prompt = min(max(prompt_len[b], 0), len(text)) if prompt_len is not None and history is not None else 0
                given = text[prompt:] + ([int(t) for t in tokens[row_off[b]:r + 1]] if tokens is not None else [])
                for v in {t for t in text[:prompt] + given if 0 <= t < vocab}:
                    y[v] = y[v] / rho if y[v] > 0 else y[v] * rho
                times = {}
                for t in given:
                    times[t] = times.get(t, 0) + 1
                for v, n in times.items():
                    if 0 <= v < vocab:
                        y[v] = y[v] - (alpha + beta * n)
            if biases is not None:
                for v, value in dict(biases[b]).items():           # the last of several
                    if 0 <= v < vocab:
                        y[v] += value
            if mask is not None:
                m = r if mask_row is None else mask_row[r]
                if 0 <= m < len(mask):
                    y[~np.asarray(mask[m][:vocab], bool)] = -np.inf
            out[r] = y
    return out
