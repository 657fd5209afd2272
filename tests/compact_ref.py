"""Plain numpy references, in 64 bits, of the calls that keep a cache small: the 4-bit format, decode over it, gathered
attention weights, eviction.  Written from the definitions in include/gva.h; they share no code with the library."""
import numpy as np


def quantise(x):
    """Rows x [..., d] (float32) -> (codes uint8 [..., d], step float16 [...], lowest float16 [...])."""
    bad = np.isnan(x).any(axis=-1)
    x = np.clip(np.where(np.isnan(x), np.float32(0), x), np.float32(-65504), np.float32(65504)).astype(np.float64)
    low = x.min(axis=-1)
    z = low.astype(np.float16)
    z = np.where(z.astype(np.float64) > low, np.nextafter(z, np.float16(-np.inf)), z)
    high = x.max(axis=-1)
    s = ((high - z.astype(np.float64)) / 15).astype(np.float16)
    with np.errstate(over="ignore"):
        while True:
            short = z.astype(np.float64) + 15 * s.astype(np.float64) < high
            if not short.any():
                break
            s = np.where(short, np.nextafter(s, np.float16(np.inf)), s)
        while True:
            less = np.nextafter(s, np.float16(-np.inf))
            roomy = (s > 0) & (z.astype(np.float64) + 15 * less.astype(np.float64) >= high)
            if not roomy.any():
                break
            s = np.where(roomy, less, s)
    c = np.zeros(x.shape, dtype=np.uint8)
    sd, zd = s.astype(np.float64)[..., None], z.astype(np.float64)[..., None]
    for k in range(15):
        c += ((x >= zd + (k + 0.5) * sd) & (sd > 0)).astype(np.uint8)
    c[bad] = 0
    return c, np.where(bad, np.float16(0), s).astype(np.float16), np.where(bad, np.float16(np.nan), z).astype(np.float16)


def widen(c, s, z):
    return z.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * c.astype(np.float64)


def pack(c):
    """Codes [..., d] -> bytes [..., d / 2]: dim 2 i in the low nibble."""
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def unpack(b):
    return np.stack([b & 15, b >> 4], axis=-1).reshape(*b.shape[:-1], 2 * b.shape[-1])


def rotate(x, pos, base=10000.0):
    x, pos = np.asarray(x, dtype=np.float64), np.asarray(pos, dtype=np.float64)
    d = x.shape[-1]
    y = np.empty_like(x)
    for i in range(d // 2):
        a = pos * base ** (-2.0 * i / d)
        y[..., 2 * i] = x[..., 2 * i] * np.cos(a) - x[..., 2 * i + 1] * np.sin(a)
        y[..., 2 * i + 1] = x[..., 2 * i] * np.sin(a) + x[..., 2 * i + 1] * np.cos(a)
    return y


def to_bf16_bits(y):
    """float64 -> bf16 bit patterns, rounded once, to nearest even (by way of f32 one in 2^17 numbers would be rounded twice)."""
    y = np.asarray(y, dtype=np.float64)
    u = y.astype(np.float32).view(np.uint32) & np.uint32(0x7FFFFFFF)
    low = u & np.uint32(0xFFFF0000)                       # the bf16 numbers on both sides of |y|
    middle = (low | np.uint32(0x8000)).view(np.float32).astype(np.float64)
    up = (np.abs(y) > middle) | ((np.abs(y) == middle) & ((low >> 16) & 1 == 1))
    return ((low >> 16) + up + np.where(np.signbit(y), 0x8000, 0)).astype(np.uint16)


def rows_of(pool, table, b, n, page):
    """Rows of slots 0 .. n - 1 of sequence b: pool [pages][G][page][d] -> [n][G][d], or [pages][page][d] -> [n][d]."""
    t = np.arange(n)
    ids = table[b, t // page] if table is not None else None
    if pool.ndim == 4:
        return pool[ids, :, t % page]
    return pool[ids, t % page]


def scores(q, v, kr, scale):
    """q [R][H][d_q], v [n][G][d_v], kr [n][d_r] -> scaled scores [R][H][n]."""
    R, H, _ = q.shape
    G, d_v = v.shape[1:]
    out = np.empty((R, H, v.shape[0]))
    for h in range(H):
        out[:, h] = q[:, h, :d_v] @ v[:, h // (H // G)].T + q[:, h, d_v:] @ kr.T
    return out * scale


def attend(q, v, kr, scale):
    """q [H][d_q] over all rows -> (out [H][d_v], lse [H]); no rows: zeros and -inf."""
    H = q.shape[0]
    G, d_v = v.shape[1:]
    if v.shape[0] == 0:
        return np.zeros((H, d_v)), np.full(H, -np.inf)
    x = scores(q[None], v, kr, scale)[0]
    top = x.max(axis=-1, keepdims=True)
    p = np.exp(x - top)
    total = p.sum(axis=-1, keepdims=True)
    out = np.stack([(p[h] / total[h]) @ v[:, h // (H // G)] for h in range(H)])
    return out, (top + np.log(total))[:, 0]


def gathered(q, lse, v, kr, scale, before, decay):
    """q [R][H][d_q], lse [R][H]: row i of R sees n - (R - 1 - i) of the n rows."""
    n, R = v.shape[0], q.shape[0]
    w = decay * before.astype(np.float64) if decay else np.zeros(n)
    x = scores(q, v, kr, scale)
    for r in range(R):
        m = n - (R - 1 - r)
        if m > 0:
            live = ~np.isneginf(lse[r])
            w[:m] += np.exp(x[r, live, :m] - lse[r, live, None]).sum(axis=0)
    return w


def evict(w, pos, keep, next_pos, sinks, recent):
    """One sequence: weights and positions [n] -> (moves [(to, from)], weights [n], positions [n]) after the eviction."""
    n = len(w)
    keep = min(keep, n)

    def key(t):
        safe = pos[t] < sinks or pos[t] >= next_pos - recent
        return np.inf if safe else (-np.inf if np.isnan(w[t]) else float(w[t]))

    stay = set(sorted(range(n), key=lambda t: (-key(t), t))[:keep])
    holes = [t for t in range(keep) if t not in stay]
    behind = [t for t in range(keep, n) if t in stay]
    assert len(holes) == len(behind)
    new_w, new_p = np.zeros(n, dtype=w.dtype), np.full(n, -1, dtype=np.int32)
    for t in range(keep):
        if t in stay:
            new_w[t], new_p[t] = w[t], pos[t]
    for to, t in zip(holes, behind):
        new_w[to], new_p[to] = w[t], pos[t]
    return list(zip(holes, behind)), new_w, new_p
