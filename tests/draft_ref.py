"""Plain references, in 64 bits or in whole numbers, of the calls around a step with drafted tokens."""
import numpy as np


def assign_pages(used, want, pages, table, P, num_pages, ring, free, max_rows):
    """What gva_assign_pages leaves: dict of its outputs (ring and table as new arrays), one sequence after the other."""
    table, ring, out_pages, lens = table.copy(), ring.copy(), list(pages), list(used)
    B, most = table.shape
    first, count = free
    fit = lambda b: used[b] >= 0 and want[b] >= 0 and 0 <= pages[b] <= most and want[b] <= most * P and used[b] <= pages[b] * P  # noqa: E731
    sound = 0 <= first < num_pages and 0 <= count <= num_pages
    code = 0 if sound else 5
    cu, pos, slots, taken, back, open_ = [0], [], [], 0, [], True
    for b in range(B):
        rows = 0
        if sound and not fit(b):
            code = code or 6
        elif sound:
            to = -(-want[b] // P)
            grow = max(want[b] - used[b], 0)
            take = max(to - pages[b], 0)
            if grow and open_ and (taken + take > count or len(pos) + grow > max_rows):
                open_ = False
            if grow and not open_:
                code = code or 9
            else:
                rows, lens[b], out_pages[b] = grow, want[b], to
                for j in range(pages[b], to):
                    table[b, j] = ring[(first + taken) % num_pages]
                    taken += 1
                back += [table[b, j] for j in range(to, pages[b])]
        for i in range(rows):
            t = used[b] + i
            page = table[b, t // P]
            pos.append(t)
            slots.append(page * P + t % P if 0 <= page < num_pages else -1)
        cu.append(cu[-1] + rows)
    free_out = list(free)
    if sound:
        for i, page in enumerate(back[: num_pages - count]):
            ring[(first + count + i) % num_pages] = page
        free_out = [(first + taken) % num_pages, count - taken + min(len(back), num_pages - count)]
        if len(back) > num_pages - count:
            code = code or 5
    return {"pages": out_pages, "lens": lens, "cu": cu, "pos": pos, "slots": slots, "table": table, "ring": ring, "free": free_out, "code": code}


def ancestors(parents):
    """What each node of one tree sees of it: [n][n] truth values."""
    n = len(parents)
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        at = i
        while at >= 0:
            see[i, at] = True
            at = parents[at]
    return see


def mask_words(see, words):
    """[n][m] truth values as [n][words] words of 32 bits."""
    bits = np.zeros((see.shape[0], words * 32), dtype=np.uint8)
    bits[:, : see.shape[1]] = see
    return np.packbits(bits, axis=1, bitorder="little").view(np.uint32).reshape(see.shape[0], words)


def commit(parents, tokens, chosen):
    """(nodes that stay, the token chosen after the last of them) of one tree."""
    path = []
    at = 0 if len(parents) else None
    while at is not None:
        path.append(at)
        at = next((i for i in range(len(parents)) if parents[i] == path[-1] and tokens[i] == chosen[path[-1]]), None)
    return path, (int(chosen[path[-1]]) if path else -1)


def frequencies(d_rot, base=10000.0, scaling="plain", factor=1.0, low=0.0, high=0.0, original_len=0):
    i = np.arange(d_rot // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (d_rot / (d_rot - 2))
    f = base ** (-2 * i / d_rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        g = np.clip((original_len * f / (2 * np.pi) - low) / (high - low), 0, 1)
        f = g * f + (1 - g) * f / factor
    return f


def rotate(x, pos, f, halves, magnitude=1.0):
    """x [n][heads][d] with the first 2 len(f) elements rotated to pos [n]."""
    y, d = x.astype(np.float64).copy(), 2 * len(f)
    a = np.asarray(pos, dtype=np.float64)[:, None, None] * f
    c, s = magnitude * np.cos(a), magnitude * np.sin(a)
    lo, hi = (slice(0, d // 2), slice(d // 2, d)) if halves else (slice(0, d, 2), slice(1, d, 2))
    u, v = x[..., lo].astype(np.float64), x[..., hi].astype(np.float64)
    y[..., lo], y[..., hi] = u * c - v * s, u * s + v * c
    return y


def tree_attention(q, v, kr, see, ctx, scale, G):
    """q [n][H][d_v + d_r], v [T][G][d_v], kr [T][d_r] in 64 bits, see [n][m] -> out, lse, sum of weight * |value|, sum of |q| |k| at most."""
    n, H, _ = q.shape
    d_v, T = v.shape[2], v.shape[0]
    vis = np.ones((n, T), dtype=bool)
    vis[:, ctx:] = see[:, : T - ctx]
    out, lse, size, terms = np.zeros((n, H, d_v)), np.full((n, H), -np.inf), np.zeros((n, H, d_v)), 0.0
    for h in range(H):
        k = np.concatenate([v[:, h // (H // G)], kr], axis=1)
        s = (q[:, h] @ k.T) * scale
        terms = max(terms, float((np.abs(q[:, h]) @ np.abs(np.nan_to_num(k, posinf=0, neginf=0)).T).max(initial=0.0)) * scale)
        for i in range(n):
            if vis[i].any():
                x, y = s[i, vis[i]], v[vis[i], h // (H // G)]
                top = x.max()
                p = np.exp(x - top)
                lse[i, h] = top + np.log(p.sum())
                out[i, h] = p @ y / p.sum()
                size[i, h] = p @ np.abs(y) / p.sum()
    return out, lse, size, terms
