"""Plain numpy forms of the cache held in 8 bits, of attention over it in 64 bits, of rotary positions and of block tables: what the
kernels' results are compared with. Nothing here comes from the package."""
import numpy as np

MOST = 2.0 ** 100


def values_of(code):
    """uint8 e4m3 codes -> float64."""
    code = np.asarray(code, np.int64)
    sign, e, m = np.where(code & 128, -1.0, 1.0), (code >> 3) & 15, code & 7
    x = np.where(e > 0, (8 + m) * np.exp2(e - 10.0), m * 2.0 ** -9)
    return np.where((code & 127) == 127, np.nan, sign * x)


CODES = values_of(np.arange(127))


def code_of(x):
    """float64 of at most 448 -> e4m3 codes, to the nearest, ties to the even code; the sign of a zero is kept."""
    a = np.abs(x)
    at = np.clip(np.searchsorted(CODES, a), 0, 126)
    low = np.maximum(at - 1, 0)
    d_low, d_at = a - CODES[low], CODES[at] - a
    pick = np.where(d_low < d_at, low, np.where(d_low > d_at, at, np.where(low % 2 == 0, low, at)))
    return (pick | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(most):
    """the smallest 2^e, e >= -100, with most <= 448 * 2^e; 0 for 0"""
    if most == 0:
        return 0.0
    e = -100
    while most > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def page_bytes(d, page):
    return page // 16 * (32 * d + 16)


def places(d):
    """Bytes of a block: keys [16][D] and values [16][D]."""
    i, dim = np.arange(16)[:, None], np.arange(d)[None]
    return ((i // 8) * (d // 16) + dim // 16) * 128 + i % 8 * 16 + dim % 16, 16 * d + dim * 16 + i


def append(cache, k, v, slots):
    """cache uint8 [pages][H][bytes], k and v float64 [T][H][D]; the tokens of a block as one."""
    h, d = k.shape[1:]
    size = 32 * d + 16
    page = cache.shape[2] // size * 16
    blocks = {}
    for t, s in enumerate(slots):
        if 0 <= s < cache.shape[0] * page:
            blocks.setdefault(int(s) // 16, []).append((t, int(s) % 16))
    for block, tokens in blocks.items():
        at = block * 16
        for head in range(h):
            raw = cache[at // page, head, at % page // 16 * size:][:size]
            for x, where, field in ((k, places(d)[0], 32 * d), (v, places(d)[1], 32 * d + 4)):
                scale = raw[field: field + 4].view(np.float32)
                old = 0.0 if any(p == 0 for _, p in tokens) else float(scale[0])
                begins = any(p == 0 for _, p in tokens)
                new = {p: np.clip(np.where(np.isnan(x[t, head]), 0.0, x[t, head]), -MOST, MOST) for t, p in tokens}
                now = max(old, scale_of(max(float(np.abs(y).max()) for y in new.values())))
                for p in range(16):
                    if p in new:
                        raw[where[p]] = code_of(new[p] / now if now else np.zeros(d))
                    elif now > old and not begins:
                        raw[where[p]] = code_of(values_of(raw[where[p]]) * (old / now)) if old else 0
                scale[0] = now


def held(cache, d):
    """uint8 [pages][H][bytes] -> keys, values float64 [pages][H][page tokens][D] and scales [pages][H][page tokens]"""
    pages, h, size = cache.shape
    raw = cache.reshape(pages, h, -1, 32 * d + 16)
    out = []
    for where, field in ((places(d)[0], 32 * d), (places(d)[1], 32 * d + 4)):
        scale = np.ascontiguousarray(raw[..., field: field + 4]).view(np.float32)[..., 0].astype(np.float64)
        with np.errstate(invalid="ignore"):
            x = values_of(raw[..., where]) * scale[..., None, None]
        out.append((x.reshape(pages, h, -1, d), np.repeat(scale, 16, -1)))
    return out


def bit(words, at):
    at = np.asarray(at, np.int64)
    return (words.reshape(-1)[at >> 5] >> (at & 31).astype(np.uint32)) & 1


def attend(q, cache, table, lens, unit, scale, units=None, cap=0.0, slopes=None, window=0, sink=0):
    """q float64 [B][T][Hq][D] -> dict of out, lse, weights and what tolerances need: size (sum of p |v|), top (largest p of a row), count
    (tokens of the row), reach (largest sum of |q_d k_d|, times scale), wide (largest |q| times the largest sum of |k_d|, times scale),
    high (largest |score| or |bias|), vscale (largest scale of the values)"""
    b, t, hq, d = q.shape
    pages, h = cache.shape[:2]
    group, page = hq // h, cache.shape[2] // (32 * d + 16) * 16
    most = table.shape[1] * page
    n = most // unit
    r = dict(out=np.zeros((b, t, hq, d)), size=np.zeros((b, t, hq, d)), lse=np.full((b, t, hq), -np.inf), weights=np.zeros((b, h, n)))
    r.update({x: np.zeros((b, t, hq)) for x in ("top", "count", "reach", "wide", "high", "vscale")})
    (keys, _), (vals, vscale) = held(cache, d)
    for i in range(b):
        length = int(min(max(lens[i], 0), most))
        ids = np.arange(length)
        pg = table[i][ids // page]
        good = (pg >= 0) & (pg < pages)
        for j in range(h):
            see = good.copy()
            if units is not None:
                see &= bit(units, (i * h + j) * n + ids // unit).astype(bool)
            for x in range(t):
                at = length - t + x
                ok = see & (ids <= at)
                if window:
                    ok &= (ids > at - window) | (ids < sink)
                toks = ids[ok]
                if not len(toks):
                    continue
                k, v = (y[table[i][toks // page], j, toks % page] for y in (keys, vals))
                rows = slice(j * group, (j + 1) * group)
                s = q[i, x, rows] @ k.T * scale
                high = np.abs(s)
                if cap:
                    s = cap * np.tanh(s / cap)
                if slopes is not None:
                    bias = slopes[rows, None] * (toks - at)[None]
                    high, s = np.maximum(high, np.abs(bias)), s + bias
                top = s.max(-1, keepdims=True)
                e = np.exp(s - top)
                total = e.sum(-1, keepdims=True)
                p = e / total
                r["out"][i, x, rows], r["size"][i, x, rows] = p @ v, p @ np.abs(v)
                r["lse"][i, x, rows] = (top + np.log(total))[:, 0]
                r["top"][i, x, rows], r["count"][i, x, rows] = p.max(-1), len(toks)
                r["reach"][i, x, rows] = (np.abs(q[i, x, rows]) @ np.abs(k).T * abs(scale)).max(-1)
                r["wide"][i, x, rows] = np.abs(q[i, x, rows]).max(-1) * np.abs(k).sum(-1).max() * abs(scale)
                r["high"][i, x, rows] = high.max(-1)
                r["vscale"][i, x, rows] = vscale[table[i][toks // page], j, toks % page].max()
                np.add.at(r["weights"][i, j], toks // unit, p.sum(0))
    return r


def rope(x, positions, frequencies, interleaved=False, inverse=False, scale=1.0):
    """x float64 [T][H][D]"""
    r = 2 * len(frequencies)
    angle = positions.astype(np.float64)[:, None] * frequencies[None] * (-1.0 if inverse else 1.0)
    c, s = (np.cos(angle) * scale)[:, None], (np.sin(angle) * scale)[:, None]
    y = x.copy()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., first] * s + x[..., second] * c
    return y


def tables(new, lens, table, ring, state, page, tokens):
    """One request after the other; table and ring are copied. -> dict as kvp.block_tables gives it, with table and ring"""
    table, ring = table.copy(), ring.copy()
    batch, width = table.shape
    pages = len(ring)
    head, count = int(state[0]) % pages, min(max(int(state[1]), 0), pages)
    free = [int(ring[(head + i) % pages]) for i in range(count)]
    out = dict(slots=[], positions=[], rows=[], starts=[0], page_starts=[0], granted=[], lens=[])
    asked_pages = asked_tokens = given = 0
    back = []
    for i in range(batch):
        n, have = int(new[i]), min(max(int(lens[i]), 0), width * page)
        had = -(-have // page)
        yes = n < 0
        if n < 0:
            back += [int(p) for p in table[i, :had] if 0 <= p < pages]
            have = 0
        elif have + n <= width * page:
            need = -(-(have + n) // page) - had
            asked_pages += need
            asked_tokens += n
            yes = (need == 0 or asked_pages <= count) and (n == 0 or asked_tokens <= tokens)
            if yes:
                table[i, had: had + need] = free[given: given + need]
                given += need
                for pos in range(have, have + n):
                    pg = int(table[i, pos // page])
                    out["slots"].append(pg * page + pos % page if 0 <= pg < pages else -1)
                    out["positions"].append(pos)
                    out["rows"].append(i)
                have += n
        out["granted"].append(int(yes))
        out["lens"].append(have)
        out["starts"].append(len(out["slots"]))
        out["page_starts"].append(given)
    for i, p in enumerate(back):
        ring[(head + count + i) % pages] = p
    rest = tokens - len(out["slots"])
    out["slots"] += [-1] * rest
    out["positions"] += [0] * rest
    out["rows"] += [-1] * rest
    out["state"] = [(head + given) % pages, min(count - given + len(back), pages)]
    return dict({k: np.array(v) for k, v in out.items()}, table=table, ring=ring)
