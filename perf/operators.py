"""Timed cases of the operators that stand between a model's attention and the placement search: a cache held in 4 bits, the
attention that reads it and says what weight each unit received, the access bitmaps of recorded weights, and eviction by
accumulated weight. `op` says which one a case runs:

  append  cache_append, then cache_read of the same tokens: keys and values quantised into the paged cache and read back
  attend  attend: queries of the last tokens of each sequence over the cache, all units or those of a bitmap
  select  trace_weights: the `topk` units of every (group, step) that received most weight, as access bitmaps
  evict   evict: weights accumulated with a decay, the `budget` units of every group that hold most, as bitmaps

The cache. A page holds `page` tokens (a multiple of 16) of one kv-head, as page / 16 tiles of 16 tokens, and a tile
16*D + 128*N bytes, N = D / 32 groups of 32 dims, each with an fp16 scale and an fp16 zero: x ~ zero + scale * q, q = 0..15. In
order, with i = 0..15 the token of the tile, n the group, j the dim of the group, 4-bit values low half of a byte first:
  keys    [i][j / 8][n][j % 8]                                                 4 bits each, 8*D bytes
  values  [(i / 2) % 2][j / 4][i / 4][n][i % 2][j % 4]                         4 bits each, 8*D bytes
  scales and zeros of the keys [i][n] and [i][n], of the values [i / 4][n][i % 4] and [i / 4][n][i % 4], fp16, 32*N bytes each
"""
import math

import numpy as np
import torch

own = False

F16_MAX = 65504.0
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
WEIGHT_ONE = 2.0 ** 24                       # accumulated weights are whole numbers: 2^24 stands for weight 1
WEIGHT_MOST = 128.0                          # of one step


# ---- cases -----------------------------------------------------------------------------------------------------------

def _append(tokens, kv_heads, head_dim, page, dtype, **more):
    return dict(op="append", tokens=tokens, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, **more)


def _attend(batch, length, kv_heads, group, head_dim, page, unit, queries=1, ragged=False, keep=1.0, weights=True, dtype="bf16", **more):
    return dict(op="attend", batch=batch, length=length, kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, unit=unit,
                queries=queries, ragged=ragged, keep=keep, weights=weights, dtype=dtype, **more)


def _select(groups, units_per_group, steps, topk, **more):
    return dict(op="select", groups=groups, units_per_group=units_per_group, steps=steps, topk=topk, **more)


def _evict(groups, units_per_group, steps, budget, sink, recent, decay_q, serving, **more):
    return dict(op="evict", groups=groups, units_per_group=units_per_group, steps=steps, budget=budget, sink=sink, recent=recent,
                decay_q=decay_q, serving=serving, **more)


def listed():
    return [
        # One decode step of 32 sequences, one layer of an 8B-class model: a token each, all launch and latency.
        _append(32, 8, 128, 16, "bf16", name="append step"),
        # The prompt of full_8b's length (2048 units of 16 tokens) written into the cache: streaming.
        _append(32768, 8, 128, 16, "bf16", name="append prompt"),
        # One sequence of about a thousand tokens, one layer: the smallest call of a decode loop.
        _attend(1, 1021, 8, 4, 128, 16, 16, name="attend one"),
        # A decode batch of many lengths, an idle slot among them, no weights asked for: plain serving.
        _attend(32, 8192, 8, 4, 128, 16, 16, ragged=True, weights=False, name="attend batch"),
        # One layer of long_70b: 4096 units of 32 tokens, eight queries a kv-head, the weight of every unit recorded.
        _attend(1, 131072, 8, 8, 128, 32, 32, name="attend long"),
        # The same cache length for four sequences, read where the access bitmap says so: 5% of the units, long_70b's top-k.
        _attend(4, 131072, 8, 8, 128, 32, 32, keep=0.05, name="attend sparse"),
        # Four queries a sequence (drafted tokens verified at once), heads of 64, units of one token, fp16.
        _attend(8, 4096, 8, 3, 64, 64, 1, queries=4, ragged=True, dtype="fp16", name="attend drafts"),
        # Access bitmaps of recorded weights, one layer (layer_8b): 8 groups of 2048 units, 256 steps.
        _select(8, 2048, 256, 256, name="select layer"),
        # The same for a whole model (long_70b): 640 groups of 4096 units, 64 steps, 671 MB of weights.
        _select(640, 4096, 64, 205, name="select model"),
        # Eviction in a decode step: 32 sequences of 8 kv-heads, 512 units of 16 tokens, half of them kept.
        _evict(256, 512, 1, 256, 1, 4, 65536, True, name="evict step"),
        # A recorded trace of one layer (layer_8b) walked through, decaying weights.
        _evict(8, 2048, 256, 614, 1, 8, 64881, False, name="evict layer"),
        # The same for a whole model (long_70b's groups, units, steps and capacity).
        _evict(640, 4096, 64, 409, 1, 8, 65536, False, name="evict model"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "select", "evict"])
    if op == "append":
        heads, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 256])
        return _append(_log(rng, 1, min(32768, 32768 * 8 * 128 // (heads * dim))), heads, dim, rng.choice([16, 32, 64]),
                       rng.choice(["bf16", "fp16", "fp32"]) if heads * dim <= 512 else rng.choice(["bf16", "fp16"]))
    if op == "attend":
        heads, dim, page = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 256]), rng.choice([16, 32, 64])
        length = _log(rng, 1, 131072)
        batch = _log(rng, 1, max(1, min(64, 4 * 131072 * 8 * 128 // (length * heads * dim * 2))))
        return _attend(batch, length, heads, rng.randint(1, 8), dim, page, rng.choice([1, 2, 16, page]), rng.choice([1, 1, 1, 2, 3]),
                       rng.random() < 0.5, rng.choice([1.0, 1.0, 0.4, 0.05]), rng.random() < 0.7, rng.choice(["bf16", "fp16"]))
    n = _log(rng, 8, 8192)
    steps = 1 if op == "evict" and rng.random() < 0.3 else _log(rng, 1, 256)
    groups = _log(rng, 1, max(1, min(640, 64 * 640 * 4096 // (n * steps))))
    some = max(1, int(n * rng.uniform(0.03, 0.6)))
    if op == "select":
        return _select(groups, n, steps, some)
    sink, recent = rng.randint(0, 2), rng.randint(1, 8)
    return _evict(groups, n, steps, min(n, some + sink + recent), sink, recent, rng.choice([65536, 65536, 64881, 58982]), steps == 1)


def _pages(case):
    return -(-case["length"] // case["page"])


def work(case):
    if case["op"] == "append":
        n = case["tokens"] * case["kv_heads"]
        d, e = case["head_dim"], DTYPES[case["dtype"]].itemsize
        cache = n * (d + d // 4)
        return {"bytes": 4 * n * d * e + 2 * cache + 16 * case["tokens"], "flops": 12 * n * d}
    if case["op"] == "attend":
        b, h, g, d, t = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "queries"))
        tokens = b * case["length"] * (0.56 if case["ragged"] else 1.0)
        seen = tokens * case["keep"] * h
        rows = b * t * h * g
        n = b * h * _pages(case) * case["page"] // case["unit"]
        return {"bytes": int(seen * (d + d // 4) + rows * (4 * d + 4) + (4 * n if case["weights"] else 0) + (n / 8 if case["keep"] < 1 else 0)
                             + 4 * b * _pages(case)), "flops": int(4 * seen * d * g * t)}
    units = case["groups"] * case["units_per_group"]
    if case["op"] == "select":
        return {"bytes": case["steps"] * (4 * units + units // 8), "flops": case["steps"] * units}
    more = 16 * units + (units // 8 if case["serving"] else 0)
    return {"bytes": case["steps"] * (4 * units + units // 8) + more, "flops": 3 * case["steps"] * units}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _rng(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(1_000_003 * (seed % 1_000_000_007) + 17)


def _keys_values(n, heads, dim, dtype, rng):
    """Keys with a few strong channels a head and an offset, values without: as projections of a trained model have them."""
    strong = 1.0 + 3.0 * (torch.rand(heads, dim, generator=rng, device="cuda") > 0.95)
    offset = 0.5 * torch.randn(heads, dim, generator=rng, device="cuda") * strong
    k = torch.randn(n, heads, dim, generator=rng, device="cuda") * strong + offset
    v = torch.randn(n, heads, dim, generator=rng, device="cuda")
    return k.to(dtype), v.to(dtype), strong


def _words(bits):
    """bool [..., U] -> int32 [..., ceil(U / 32)], bit u & 31 of word u >> 5."""
    u = bits.shape[-1]
    full = torch.nn.functional.pad(bits, (0, -u % 32)).view(*bits.shape[:-1], -1, 32).long()
    word = (full << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(word >= 2 ** 31, word - 2 ** 32, word).int()


def _recorded(case, rng):
    """Recorded weights [steps][U]: per group and step a softmax over units whose log-importance drifts slowly, summed over four heads."""
    s, g, n = case["steps"], case["groups"], case["units_per_group"]
    rank = torch.rand(g, n, generator=rng, device="cuda").argsort(-1)
    base = -1.1 * torch.log1p(rank.float())
    x = torch.randn(g, n, generator=rng, device="cuda")
    w = torch.empty(s, g, n, device="cuda")
    for t in range(s):
        torch.mul(torch.softmax(base + x, -1), 4.0, out=w[t])
        x = 0.95 * x + 0.3122 * torch.randn(g, n, generator=rng, device="cuda")
    return w.view(s, g * n)


def prepare(case, seed):
    rng = _rng(seed)
    if case["op"] == "append":
        n, h, d, page = case["tokens"], case["kv_heads"], case["head_dim"], case["page"]
        k, v, _ = _keys_values(n, h, d, DTYPES[case["dtype"]], rng)
        used = -(-n // page)
        pages = 2 * used + 3
        order = torch.randperm(pages, generator=rng, device="cuda")[:used]
        if n <= 256:                                            # a token of each sequence, somewhere in its last page
            pages = 4 * n + 3
            order = torch.randperm(pages, generator=rng, device="cuda")[:n]
            slots = order * page + torch.randint(0, page, (n,), generator=rng, device="cuda")
        else:
            slots = (order[:, None] * page + torch.arange(page, device="cuda")).view(-1)[:n]
        cache = torch.zeros(pages, h, page * (d + d // 4), dtype=torch.uint8, device="cuda")
        return dict(case=case, k=k, v=v, slots=slots.contiguous(), cache=cache)
    if case["op"] == "attend":
        b, h, g, d, page, t = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "page", "queries"))
        dtype, length, used = DTYPES[case["dtype"]], case["length"], _pages(case)
        pages = b * used + 5
        table = torch.randperm(pages, generator=rng, device="cuda")[: b * used].view(b, used)
        cache = torch.zeros(pages, h, page * (d + d // 4), dtype=torch.uint8, device="cuda")
        q = torch.empty(b, t, h * g, d, dtype=dtype, device="cuda")
        for i in range(b):                                      # what earlier steps left in the cache
            k, v, strong = _keys_values(used * page, h, d, dtype, rng)
            packed = _packed(k.float().view(used, page, h, d).transpose(1, 2), v.float().view(used, page, h, d).transpose(1, 2))
            cache[table[i]] = packed
            # scores with a standard deviation of about 2.5: a few units hold most of the weight
            q[i] = (2.5 * torch.randn(t, h, g, d, generator=rng, device="cuda") / strong[:, None]).reshape(t, h * g, d).to(dtype)
        lens = torch.full((b,), length, device="cuda")
        if case["ragged"]:
            lens = (length * (0.125 + 0.875 * torch.rand(b, generator=rng, device="cuda"))).long().clamp(1, length)
            lens[0] = length
            if b > 4:
                lens[-1] = 0                                    # an idle slot of the batch
        units = None
        n = used * page // case["unit"]
        if case["keep"] < 1.0:
            here = torch.arange(n, device="cuda")[None, None] * case["unit"] < lens[:, None, None]
            score = torch.rand(b, h, n, generator=rng, device="cuda").masked_fill(~here, -1.0)
            many = (case["keep"] * lens / case["unit"]).ceil().long()[:, None, None]
            keep = (score.argsort(-1, descending=True).argsort(-1) < many) & here
            units = _words(keep.view(-1))
        return dict(case=case, q=q, cache=cache, table=table.int().contiguous(), lens=lens.int(), units=units, scale=d ** -0.5)
    w = _recorded(case, rng)
    if case["op"] == "select":
        return dict(case=case, weights=w)
    u = case["groups"] * case["units_per_group"]
    state = dict(case=case, weights=w, acc=None, kept=None, exist=None)
    if case["serving"]:                                         # what earlier steps accumulated, what is left of the cache by now
        past = 30.0 * w[0] * torch.rand(u, generator=rng, device="cuda")
        state["acc"] = (past * WEIGHT_ONE).round().long()
        state["kept"] = _words(torch.rand(u, generator=rng, device="cuda") < 0.8)
        n = case["units_per_group"]
        state["exist"] = torch.randint(max(1, n // 2), n + 1, (case["groups"],), generator=rng, device="cuda").int()
    return state


# ---- the operators ---------------------------------------------------------------------------------------------------

def _quantised(x):
    """fp32 [..., D] -> q [..., N, 32] (fp32 whole numbers 0..15), scale and zero [..., N] (fp16)."""
    x = torch.nan_to_num(x, nan=0.0, posinf=F16_MAX, neginf=-F16_MAX).clamp(-F16_MAX, F16_MAX)
    x = x.view(*x.shape[:-1], -1, 32)
    low, high = x.amin(-1), x.amax(-1)
    zero = low.half()
    scale = ((high - zero.float()) / torch.full((), 15.0, device=x.device)).clamp(min=0.0).half()
    step = scale.float()[..., None]
    q = torch.where(step > 0, ((x - zero.float()[..., None]) / step).round().clamp(0, 15), torch.zeros_like(x))
    return q, scale, zero


def _nibbles(q):
    q = q.to(torch.uint8)
    return q[..., 0::2] | (q[..., 1::2] << 4)


def _packed(k, v):
    """fp32 keys and values [pages][kv_heads][page][D] -> uint8 [pages][kv_heads][page bytes], the layout at the top of the file."""
    pages, h, page, d = k.shape
    n = d // 32
    tiles = (pages, h, page // 16)
    kq, ks, kz = _quantised(k)
    vq, vs, vz = _quantised(v)
    kq = kq.view(*tiles, 16, n, 4, 8).transpose(-3, -2)
    vq = vq.view(*tiles, 4, 2, 2, n, 8, 4).permute(0, 1, 2, 4, 7, 3, 6, 5, 8)
    meta = [t.view(*tiles, 16, n) for t in (ks, kz)] + [t.view(*tiles, 4, 4, n).transpose(-1, -2) for t in (vs, vz)]
    parts = [_nibbles(kq).reshape(*tiles, -1), _nibbles(vq).reshape(*tiles, -1)]
    parts += [t.contiguous().view(torch.uint8).reshape(*tiles, -1) for t in meta]
    return torch.cat(parts, -1).reshape(pages, h, -1)


def _unpacked(tiles, d):
    """uint8 tiles [..., 16 * D + 128 * N] -> fp32 keys and values [..., 16, D]."""
    n, lead = d // 32, tiles.shape[:-1]
    ends = [8 * d, 16 * d] + [16 * d + 32 * n * i for i in (1, 2, 3, 4)]
    kq, vq, ks, kz, vs, vz = (tiles[..., a:b] for a, b in zip([0] + ends, ends))
    kq = torch.stack((kq & 15, kq >> 4), -1).view(*lead, 16, 4, n, 8).transpose(-3, -2)
    vq = torch.stack((vq & 15, vq >> 4), -1).view(*lead, 2, 8, 4, n, 2, 4)
    m = len(lead)
    vq = vq.permute(*range(m), m + 2, m, m + 4, m + 3, m + 1, m + 5)
    ks, kz = (t.contiguous().view(torch.float16).view(*lead, 16, n).float() for t in (ks, kz))
    vs, vz = (t.contiguous().view(torch.float16).view(*lead, 4, n, 4).transpose(-1, -2).reshape(*lead, 16, n).float() for t in (vs, vz))
    k = kq.reshape(*lead, 16, n, 32) * ks[..., None] + kz[..., None]
    v = vq.reshape(*lead, 16, n, 32) * vs[..., None] + vz[..., None]
    return k.reshape(*lead, 16, d), v.reshape(*lead, 16, d)


def _append_plain(s):
    cache, slots = s["cache"], s["slots"]
    h, d, page = s["case"]["kv_heads"], s["case"]["head_dim"], s["case"]["page"]
    n = d // 32
    bytes_ = torch.arange(page * (d + d // 4), device="cuda").view(page // 16, -1)
    at = slots % page
    tile, i = at // 16, at % 16
    parts = []
    for x, is_key in ((s["k"], True), (s["v"], False)):
        q, scale, zero = _quantised(x.float())                                  # [T][H][N][32], [T][H][N]
        meta = torch.stack((scale, zero), 2).view(torch.uint8).view(-1, h, 2, n, 2)
        if is_key:
            places = bytes_[:, : 8 * d].view(-1, 16, 4, n, 4).transpose(2, 3)[tile, i]
            fields = bytes_[:, 16 * d: 16 * d + 64 * n].view(-1, 2, 16, n, 2)[tile, :, i]
        else:
            places = bytes_[:, 8 * d: 16 * d].view(-1, 2, 8, 4, n, 2, 2)[tile, (i // 2) % 2, :, i // 4, :, i % 2].transpose(1, 2)
            fields = bytes_[:, 16 * d + 64 * n:].view(-1, 2, 4, n, 4, 2)[tile, :, i // 4, :, i % 4]
        parts.append((places.reshape(len(slots), 1, -1), _nibbles(q).reshape(len(slots), h, -1)))
        parts.append((fields.reshape(len(slots), 1, -1), meta.reshape(len(slots), h, -1)))
    head = torch.arange(h, device="cuda")[None, :, None]
    for where, what in parts:
        cache[(slots // page)[:, None, None], head, where] = what
    back = []
    for where, what in zip((parts[0], parts[2]), (parts[1], parts[3])):         # read what the cache holds now
        byte = cache[(slots // page)[:, None, None], head, where[0]]
        q = torch.stack((byte & 15, byte >> 4), -1).view(len(slots), h, n, 32).float()
        scale, zero = cache[(slots // page)[:, None, None], head, what[0]].view(torch.float16).view(len(slots), h, 2, n).float().unbind(2)
        back.append((q * scale[..., None] + zero[..., None]).reshape(len(slots), h, d).to(s["k"].dtype))
    return back


def _attend_plain(s):
    case, q, lens = s["case"], s["q"], s["lens"].long()
    b, h, g, d, t = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "queries"))
    tiles = s["cache"][s["table"].long()].transpose(1, 2).reshape(b, h, -1, 16 * d + 4 * d)
    k, v = (x.reshape(b, h, -1, d) for x in _unpacked(tiles, d))
    many, unit = k.shape[2], case["unit"]
    last = lens[:, None] - t + 1 + torch.arange(t, device="cuda")               # query j sees the tokens before this one
    seen = torch.arange(many, device="cuda") < last[:, :, None]                 # [B][T][tokens]
    seen = seen[:, None, :, None, :]
    if s["units"] is not None:
        u = torch.arange(b * h * (many // unit), device="cuda")
        bits = (s["units"][u >> 5].long() >> (u & 31)) & 1
        seen = seen & bits.bool().view(b, h, -1).repeat_interleave(unit, -1)[:, :, None, None, :]
    x = q.float().view(b, t, h, g, d).permute(0, 2, 1, 3, 4).reshape(b, h, t * g, d)
    score = (torch.matmul(x, k.transpose(-1, -2)) * s["scale"]).view(b, h, t, g, many).masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    out = torch.matmul(p.view(b, h, t * g, many), v).view(b, h, t, g, d).permute(0, 2, 1, 3, 4).reshape(b, t, h * g, d).to(q.dtype)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(b, t, h * g)
    found = [out, lse]
    if case["weights"]:
        found.append(p.sum((2, 3)).view(b, h, many // unit, unit).sum(-1))
    return found


def _most(keys, many, allowed):
    """Per row of `keys`: the `many` allowed entries with the largest key, ties to the lower index, as truth values."""
    order = torch.sort(keys.masked_fill(~allowed, -1), dim=-1, descending=True, stable=True).indices
    rank = torch.arange(keys.shape[-1], device=keys.device).expand_as(order)
    return torch.zeros_like(allowed).scatter_(-1, order, rank < many) & allowed


def _select_plain(s):
    case = s["case"]
    w = s["weights"].view(case["steps"], case["groups"], -1)
    return [_words(_most(w, case["topk"], w > 0).view(case["steps"], -1))]


def _evict_plain(s):
    case, w = s["case"], s["weights"]
    g, n, u = case["groups"], case["units_per_group"], w.shape[1]
    fixed = torch.round(w.clamp(0.0, WEIGHT_MOST).double() * WEIGHT_ONE).long()
    acc = s["acc"] if s["acc"] is not None else torch.zeros(u, dtype=torch.int64, device="cuda")
    past = []
    for row in fixed:                                                           # the recurrence: each step needs the one before
        acc = ((acc * case["decay_q"]) >> 16) + row
        past.append(acc)
    held = torch.stack(past).view(-1, g, n)
    unit = torch.arange(n, device="cuda")[None]
    exist = s["exist"].long()[:, None] if s["exist"] is not None else torch.full((g, 1), n, device="cuda")
    safe = ((unit < case["sink"]) | (unit >= exist - case["recent"])) & (unit < exist)
    old = torch.ones(g, n, dtype=torch.bool, device="cuda")
    if s["kept"] is not None:
        bit = torch.arange(u, device="cuda")
        old = ((s["kept"][bit >> 5].long() >> (bit & 31)) & 1).bool().view(g, n)
    left = (case["budget"] - safe.sum(-1, keepdim=True)).clamp(min=0)
    allowed = (old & ~safe & (unit < exist)).expand_as(held)
    return [_words((_most(held, left, allowed) | safe).view(held.shape[0], -1)), acc]


def run(s):
    case = s["case"]
    if own:
        from paper_2508_13231_b200 import kvp
        if case["op"] == "append":
            kvp.cache_append(s["cache"], s["k"], s["v"], s["slots"])
            return list(kvp.cache_read(s["cache"], s["slots"], case["head_dim"], s["k"].dtype))
        if case["op"] == "attend":
            r = kvp.attend(s["q"], s["cache"], s["table"], s["lens"], unit_tokens=case["unit"], scale=s["scale"], units=s["units"],
                           want_lse=True, want_weights=case["weights"])
            return [r["out"], r["lse"]] + ([r["weights"]] if case["weights"] else [])
        if case["op"] == "select":
            return [kvp.trace_weights(s["weights"], case["groups"], case["topk"])]
        r = kvp.evict(s["weights"], case["groups"], case["budget"], sink=case["sink"], recent=case["recent"], decay_q=case["decay_q"],
                      acc=s["acc"], kept=s["kept"], exist=s["exist"])
        return [r["kept"], r["acc"]]
    if case["op"] == "append":
        return _append_plain(s)
    if case["op"] == "attend":
        return _attend_plain(s)
    return _select_plain(s) if case["op"] == "select" else _evict_plain(s)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _rounded(x):
    """What the 4-bit form keeps of x [..., D]: the group's lowest value and a fifteenth of its range, both in fp16, and whole steps."""
    x = x.double().unflatten(-1, (-1, 32))
    lo = x.min(-1, keepdim=True).values.half().double()
    st = ((x.max(-1, keepdim=True).values - lo) / 15).half().double()
    q = torch.round((x - lo) / torch.where(st > 0, st, 1.0)).clamp(0, 15) * (st > 0)
    return (lo + st * q).flatten(-2)


def _held(page_bytes, d):
    """One kv-head's pages of one sequence [pages][bytes] -> keys and values [tokens][D] in 64 bits, a field at a time."""
    n, dev = d // 32, page_bytes.device
    tile = page_bytes.reshape(-1, 20 * d)
    i, dim = torch.arange(16, device=dev)[:, None], torch.arange(d, device=dev)[None]
    grp, j = dim // 32, dim % 32
    kn = ((i * 4 + j // 8) * n + grp) * 8 + j % 8
    vn = (((((i // 2) % 2 * 8 + j // 4) * 4 + i // 4) * n + grp) * 2 + i % 2) * 4 + j % 4
    half = tile[:, 16 * d:].contiguous().view(torch.float16).double()
    ki, vi = i * n + grp, (i // 4 * n + grp) * 4 + i % 4
    out = []
    for at, first, sc in ((kn, 0, ki), (vn, 8 * d, vi + 32 * n)):
        q = (tile[:, first + at // 2].long() >> (4 * (at % 2))) & 15
        out.append((half[:, sc + 16 * n] + half[:, sc] * q).reshape(-1, d))
    return out


def exact(case, seed):
    if case["op"] == "append":
        s = prepare(case, seed)
        return [_rounded(s["k"]), _rounded(s["v"])]
    if case["op"] != "attend":
        return None                                             # whole numbers: they have to be equal
    s = prepare(case, seed)
    b, h, g, d, t, unit = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "queries", "unit"))
    many = _pages(case) * case["page"]
    n = many // unit
    out = torch.zeros(b, t, h * g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, t, h * g), -math.inf, dtype=torch.float64, device="cuda")
    got = torch.zeros(b, h, n, dtype=torch.float64, device="cuda")
    words = None if s["units"] is None else np.unpackbits(s["units"].cpu().numpy().view(np.uint8), bitorder="little")[: b * h * n].reshape(b, h, n)
    for i in range(b):
        length = int(s["lens"][i])
        for j in range(h):
            k, v = _held(s["cache"][s["table"][i].long(), j], d)
            for r in range(t):
                ids = torch.arange(max(0, length - t + 1 + r), device="cuda")
                if words is not None:
                    ids = ids[torch.from_numpy(words[i, j]).cuda()[ids // unit] > 0]
                if not len(ids):
                    continue
                x = s["q"][i, r, j * g: (j + 1) * g].double() @ k[ids].T * s["scale"]
                lse[i, r, j * g: (j + 1) * g] = torch.logsumexp(x, -1)
                p = torch.softmax(x, -1)
                out[i, r, j * g: (j + 1) * g] = p @ v[ids]
                got[i, j].index_add_(0, ids // unit, p.sum(0))
    return [out, lse] + ([got] if case["weights"] else [])
