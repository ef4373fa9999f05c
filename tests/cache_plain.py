"""Plain numpy forms of the cache held in 4 bits, of attention over it in 64 bits, of the selection by weight and of eviction:
what the kernels' results are compared with. Nothing here comes from the package."""
import numpy as np

F16_MAX = np.float32(65504)


def quantised(x):
    """float32 [..., D] -> q uint8 [..., N, 32], scale and zero float16 [..., N], one fp32 operation at a time."""
    x = np.where(np.isnan(x), np.float32(0), x).astype(np.float32)
    x = (np.clip(x, -F16_MAX, F16_MAX) + np.float32(0)).reshape(*x.shape[:-1], -1, 32)
    low, high = x.min(-1), x.max(-1)
    zero = low.astype(np.float16)
    z = zero.astype(np.float32)
    scale = np.maximum((high - z) / np.float32(15), np.float32(0)).astype(np.float16)
    s = scale.astype(np.float32)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(s > 0, np.rint((x - z[..., None]) / s), 0)
    return np.clip(q, 0, 15).astype(np.uint8), scale, zero


def places(d):
    """Where a tile keeps things: 4-bit numbers of keys and values [16][D] (number of the 4 bits), scales and zeros of keys and
    values, four times [16][N] (byte)."""
    n = d // 32
    i, dim = np.arange(16)[:, None], np.arange(d)[None]
    g, j = dim // 32, dim % 32
    key = ((i * 4 + j // 8) * n + g) * 8 + j % 8
    value = 16 * d + (((((i // 2) % 2 * 8 + j // 4) * 4 + i // 4) * n + g) * 2 + i % 2) * 4 + j % 4
    grp = np.arange(n)[None]
    by_token, by_four = (i * n + grp) * 2, ((i // 4 * n + grp) * 4 + i % 4) * 2
    at = 16 * d
    return key, value, [at + by_token, at + 32 * n + by_token, at + 64 * n + by_four, at + 96 * n + by_four]


def page_bytes(d, page):
    return page // 16 * 20 * d


def put(cache, slot, k, v):
    """Writes one token: cache uint8 [pages][H][bytes], k and v float32 [H][D]."""
    h, d = k.shape
    page = cache.shape[2] // (20 * d) * 16
    if slot < 0 or slot >= cache.shape[0] * page:
        return
    key, value, meta = places(d)
    i = slot % 16
    for head in range(h):
        tile = cache[slot // page, head, slot % page // 16 * 20 * d:][: 20 * d]
        for x, where, (ms, mz) in ((k, key, (meta[0], meta[1])), (v, value, (meta[2], meta[3]))):
            q, scale, zero = quantised(x[head])
            at, q = where[i], q.reshape(-1)
            for low in (0, 1):
                sel = at % 2 == low
                byte = at[sel] // 2
                tile[byte] = (tile[byte] & (0xF0 if low == 0 else 0x0F)) | (q[sel] << (4 * low))
            for m, field in ((ms[i], scale), (mz[i], zero)):
                raw = field.view(np.uint8).reshape(-1, 2)
                tile[m], tile[m + 1] = raw[:, 0], raw[:, 1]


def tile_values(tile, d):
    """uint8 [tiles][20 D] -> (q, scale, zero) of the keys and of the values, float64 [tiles][16][D]."""
    key, value, meta = places(d)
    grp = np.arange(d) // 32
    out = []
    for where, (ms, mz) in ((key, meta[:2]), (value, meta[2:])):
        q = (tile[:, where // 2] >> (4 * (where % 2)).astype(np.uint8)) & 15
        f16 = [np.ascontiguousarray(np.stack([tile[:, m], tile[:, m + 1]], -1)).view(np.float16)[..., 0].astype(np.float64)[..., grp] for m in (ms, mz)]
        out.append((q.astype(np.float64), *f16))
    return out


def read(cache, slot, d):
    """-> k, v float32 [H][D] as the cache holds them."""
    page = cache.shape[2] // (20 * d) * 16
    h = cache.shape[1]
    if slot < 0 or slot >= cache.shape[0] * page:
        return np.zeros((h, d), np.float32), np.zeros((h, d), np.float32)
    at = slot % page // 16 * 20 * d
    out = []
    for q, s, z in tile_values(cache[slot // page, :, at: at + 20 * d], d):
        out.append((q[:, slot % 16].astype(np.float32) * s[:, slot % 16].astype(np.float32)).astype(np.float32) + z[:, slot % 16].astype(np.float32))
    return out


def bit(words, at):
    at = np.asarray(at, np.int64)
    return (words.reshape(-1)[at >> 5] >> (at & 31).astype(np.uint32)) & 1


def attend(q, cache, table, lens, unit, scale, units=None):
    """q float64 [B][T][Hq][D], cache uint8 [pages][H][bytes] -> dict of out, lse, weights and what tolerances need:
    size (sum of p |value|, the values as |zero| + scale q), top (largest p of a row), count (tokens of the row),
    reach (largest sum of |q_d| (|zero| + scale q) of a row, times scale)."""
    b, t, hq, d = q.shape
    pages, h = cache.shape[:2]
    group, page = hq // h, cache.shape[2] // (20 * d) * 16
    most = table.shape[1] * page
    n = most // unit
    r = dict(out=np.zeros((b, t, hq, d)), size=np.zeros((b, t, hq, d)), lse=np.full((b, t, hq), -np.inf), weights=np.zeros((b, h, n)),
             top=np.zeros((b, t, hq)), count=np.zeros((b, t, hq)), reach=np.zeros((b, t, hq)), vscale=np.zeros((b, t, hq)))
    for i in range(b):
        length = int(min(max(lens[i], 0), most))
        ids = np.arange(length)
        good = (table[i][ids // page] >= 0) & (table[i][ids // page] < pages)
        for j in range(h):
            see = good.copy()
            if units is not None:
                see &= bit(units, (i * h + j) * n + ids // unit).astype(bool)
            toks = ids[see]
            if not len(toks):
                continue
            used = np.unique(toks // 16)
            raw = np.stack([cache[table[i][u * 16 // page], j, u * 16 % page // 16 * 20 * d:][: 20 * d] for u in used])
            (kq, ks, kz), (vq, vs, vz) = tile_values(raw, d)
            pick = (np.searchsorted(used, toks // 16), toks % 16)
            kq, ks, kz, vq, vs, vz = (x[pick] for x in (kq, ks, kz, vq, vs, vz))
            k, v = kz + ks * kq, vz + vs * vq
            kabs, vabs = np.abs(kz) + ks * kq, np.abs(vz) + vs * vq
            for x in range(t):
                mine = toks < length - t + 1 + x
                if not mine.any():
                    continue
                rows = slice(j * group, (j + 1) * group)
                s = q[i, x, rows] @ k[mine].T * scale
                top = s.max(-1, keepdims=True)
                e = np.exp(s - top)
                total = e.sum(-1, keepdims=True)
                p = e / total
                r["out"][i, x, rows] = p @ v[mine]
                r["size"][i, x, rows] = p @ vabs[mine]
                r["lse"][i, x, rows] = (top + np.log(total))[:, 0]
                r["top"][i, x, rows] = p.max(-1)
                r["count"][i, x, rows] = mine.sum()
                r["reach"][i, x, rows] = (np.abs(q[i, x, rows]) @ kabs[mine].T * abs(scale)).max(-1)
                r["vscale"][i, x, rows] = vs[mine].max()
                np.add.at(r["weights"][i, j], toks[mine] // unit, p.sum(0))
    return r


def most_of(key, many, allowed):
    """The `many` allowed entries with the largest key, ties to the lower index."""
    order = np.argsort(-np.asarray(key, np.float64 if np.asarray(key).dtype.kind == "f" else np.int64), kind="stable")
    out = np.zeros(len(order), bool)
    out[order[np.asarray(allowed)[order]][:many]] = True
    return out


def pack(bits):
    """bool [..., U] -> uint32 [..., ceil(U / 32)]."""
    u = bits.shape[-1]
    full = np.zeros(bits.shape[:-1] + (-(-u // 32) * 32,), np.uint8)
    full[..., :u] = bits
    return np.packbits(full, axis=-1, bitorder="little").view(np.uint32)


def select(weights, groups, topk):
    s, u = weights.shape
    w = weights.reshape(s, groups, -1)
    out = np.zeros(w.shape, bool)
    for a in range(s):
        for g in range(groups):
            ok = w[a, g] > 0
            out[a, g] = most_of(np.where(ok, w[a, g], 0), topk, ok)
    return pack(out.reshape(s, u))


def evict(weights, groups, budget, sink, recent, decay_q, acc=None, kept=None, exist=None, before=False):
    s, u = weights.shape
    n = u // groups
    most = np.uint64(2 ** 48 - 1)
    a = np.zeros(u, np.uint64) if acc is None else np.minimum(np.maximum(np.asarray(acc, np.int64), 0).astype(np.uint64), most)
    old = np.ones(u, bool) if kept is None else bit(kept, np.arange(u)).astype(bool)
    fixed = np.rint(np.clip(np.nan_to_num(weights.astype(np.float64), nan=0.0, posinf=128.0), 0, 128) * 2.0 ** 24).astype(np.uint64)
    out = np.zeros((s, u), bool)

    def choose(row):
        for g in range(groups):
            e = n if exist is None else min(max(int(exist[g]), 0), n)
            i = np.arange(n)
            safe = ((i < sink) | (i >= e - recent)) & (i < e)
            allowed = old[g * n:(g + 1) * n] & ~safe & (i < e)
            row[g * n:(g + 1) * n] = safe | most_of(a[g * n:(g + 1) * n].astype(np.int64), max(0, budget - int(safe.sum())), allowed)

    for t in range(s):
        if before:
            choose(out[t])
        if decay_q != 65536:                                  # below 2^48 * 65536: 64 bits hold the product
            a = (a * np.uint64(decay_q)) >> np.uint64(16)
        a = np.minimum(a + fixed[t], most)
        if not before:
            choose(out[t])
    return pack(out), a.astype(np.int64)
