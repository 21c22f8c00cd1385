"""Plain statement of the paged 4-bit cache (include/mustdrop.h, mustdrop_page_*), in numpy and 64 bits.

Rows are float64 arrays of numbers that bf16 holds; a pool is uint8 [n_pages, heads, page / 16, 20 D], a slot
page id * page + place.  Loops over tokens and sequences: small sizes only.
"""
import numpy as np


def to_bf16(x):
    """Nearest bf16 (ties to even) of numbers, as float64."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    nan = np.isnan(np.asarray(x, dtype=np.float32))
    return np.where(nan, np.nan, r.view(np.float32).astype(np.float64))


def bf16_bits(x):
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def bits_bf16(b):
    return (np.asarray(b).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def quantise(x):
    """Codes [.., D], scales and centres [.., D / 32] of rows [.., D]."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore", over="ignore"):
        fine = np.isfinite(g).all(-1)
        f = np.where(fine[..., None], g, 0.0)
        low, high = f.min(-1), f.max(-1)
        s = to_bf16((high / 2 - low / 2) / 7.5)
        z = to_bf16(low + 8 * s)
        d = np.where(s > 0, s, 1.0)[..., None]
        c = np.where(s[..., None] > 0, np.clip(np.rint((f - z[..., None]) / d) + 8, 0, 15), 8)
    s = np.where(fine, s, np.nan)
    z = np.where(fine, z, 0.0)
    c = np.where(fine[..., None], c, 0)
    return c.reshape(x.shape).astype(np.uint8), s, z


def values(c, s, z):
    v = z[..., None] + s[..., None] * (c.reshape(*c.shape[:-1], -1, 32).astype(np.float64) - 8)
    return v.reshape(c.shape)


def _places(d):
    """Byte and half of every (token, channel) of a chunk for K and V, byte of every (token, group)'s K scale, K centre, V scale, V centre."""
    k, v, meta = np.zeros((16, d, 2), int), np.zeros((16, d, 2), int), np.zeros((16, d // 32, 4), int)
    groups = d // 32
    for tok in range(16):
        r = tok // 2 + 8 * (tok % 2)
        for ch in range(d):
            g, w = divmod(ch, 32)
            t, b = divmod(w, 8)
            k[tok, ch] = ((r * 4 + t) * groups + g) * 4 + b // 2, ch % 2
            a, h = divmod(g, 2)
            i, e = divmod(w, 4)
            v[tok, ch] = 8 * d + ((((a * 8 + i) * 4 + tok // 4) * 2 + h) * 2 + e // 2) * 4 + tok % 4, ch % 2
        for g in range(groups):
            meta[tok, g] = 16 * d + 2 * (r * 2 * groups + g), 16 * d + 2 * (r * 2 * groups + groups + g), \
                18 * d + 2 * (r * groups + g), 19 * d + 2 * (g * 16 + r)
    return k, v, meta


def store(pool, slots, k, v):
    """Writes rows [n_seq, heads, rows, D] to the pool, in place."""
    page, d = 16 * pool.shape[2], pool.shape[3] // 20
    pk, pv, meta = _places(d)
    ck, sk, zk = quantise(k)
    cv, sv, zv = quantise(v)
    for s in range(slots.shape[0]):
        for r in range(slots.shape[1]):
            slot = int(slots[s, r])
            if slot < 0 or slot >= pool.shape[0] * page:
                continue
            tok = slot % 16
            for h in range(pool.shape[1]):
                c = pool[slot // page, h, slot % page // 16]
                for place, codes in ((pk[tok], ck[s, h, r]), (pv[tok], cv[s, h, r])):
                    low, high = place[0::2, 0], codes[0::2] | (codes[1::2] << 4)
                    c[low] = high
                for j, x in enumerate((sk, zk, sv, zv)):
                    b = bf16_bits(x[s, h, r])
                    c[meta[tok, :, j]], c[meta[tok, :, j] + 1] = b & 255, b >> 8


def token(pool, slot, head):
    """K and V of one stored token, float64 [D]."""
    page, d = 16 * pool.shape[2], pool.shape[3] // 20
    pk, pv, meta = _PLACES.setdefault(d, _places(d))
    c, tok = pool[slot // page, head, slot % page // 16], slot % 16
    out = []
    for place, j in ((pk[tok], 0), (pv[tok], 2)):
        codes = (c[place[:, 0]] >> (4 * place[:, 1])) & 15
        s, z = (bits_bf16(c[meta[tok, :, j + i]].astype(np.uint16) | (c[meta[tok, :, j + i] + 1].astype(np.uint16) << 8)) for i in (0, 1))
        out.append(values(codes, s, z))
    return out


_PLACES = {}


def load(pool, slots, k_out, v_out):
    """Values of stored tokens into k_out, v_out [n_seq, heads, rows, D] (float64, unrounded), in place."""
    page = 16 * pool.shape[2]
    for s, r in np.ndindex(*slots.shape):
        if 0 <= slots[s, r] < pool.shape[0] * page:
            for h in range(pool.shape[1]):
                k_out[s, h, r], v_out[s, h, r] = token(pool, int(slots[s, r]), h)


def tables(add, lens, state, ring, table, page, rows):
    """-> (len_out, state_out, ring, table, slots, refused for length, refused for pages)."""
    ring, table = ring.copy(), table.copy()
    n_pages, most = len(ring), table.shape[1] * page
    head, count = int(state[0]), int(state[1])
    len_out, slots = lens.copy(), np.full((len(lens), rows), -1, np.int32)
    asked = taken = back = 0
    bad, short = [], []
    old_ring, old_table = ring.copy(), table.copy()
    for s, (a, n) in enumerate(zip(add.tolist(), lens.tolist())):
        if n < 0 or n > most or a > rows or n + a > most:
            bad.append(s)
            continue
        had = -(-n // page)
        if a < 0:
            left = max(0, n + a)
            for e in range(-(-left // page), had):
                ring[(head + count + back) % n_pages] = old_table[s, e]
                back += 1
            len_out[s] = left
            continue
        need = -(-(n + a) // page) - had
        if need > 0 and asked + need > count:
            asked += need
            short.append(s)
            continue
        for i in range(need):
            table[s, had + i] = old_ring[(head + asked + i) % n_pages]
        asked += need
        taken = asked if need > 0 else taken
        len_out[s] = n + a
        for t in range(a):
            slots[s, t] = table[s, (n + t) // page] * page + (n + t) % page
    return len_out, np.array([(head + taken) % n_pages, count - taken + back], np.int32), ring, table, slots, bad, short


def attend(q, pool, table, lens, causal=True, scale=None):
    """q float64 [n_seq, n_q, q_heads, D] -> out likewise."""
    n, n_q, q_heads, d = q.shape
    heads, page, n_pages = pool.shape[1], 16 * pool.shape[2], pool.shape[0]
    group = q_heads // heads
    scale = d ** -0.5 if not scale else scale
    out = np.zeros(q.shape)
    for s in range(n):
        length = min(max(int(lens[s]), 0), table.shape[1] * page)
        at = [(x, int(table[s, x // page]) * page + x % page) for x in range(length) if 0 <= table[s, x // page] < n_pages]
        for h in range(heads):
            kv = [token(pool, slot, h) for _, slot in at]
            for t in range(n_q):
                limit = length - n_q + 1 + t if causal else length
                seen = [i for i, (x, _) in enumerate(at) if x < limit]
                if not seen:
                    continue
                k, v = (np.stack([kv[i][j] for i in seen]) for j in (0, 1))
                for j in range(h * group, (h + 1) * group):
                    z = k @ q[s, t, j] * scale
                    p = np.exp(z - z.max())
                    out[s, t, j] = p @ v / p.sum()
    return out
