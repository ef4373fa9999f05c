"""Timed cases of what a decode step does around a cache held in 8 bits. `op` says which operator a case runs:

  tables  block_tables: pages for the new tokens of every request, their slots and positions, pages of finished requests given back
  rope    rope: rotary positions of queries and keys, or the same turned back (the gradient)
  append  cache8_append, then cache8_read of the blocks written to: keys and values into the paged cache, a scale a block and head
  attend  attend8: queries of the last tokens of each sequence over the cache; capped scores, a bias by distance, a window

The cache. A page holds `page` tokens (a multiple of 16) of one kv-head as page / 16 blocks of 16 tokens, a block 32*D + 16 bytes.
x ~ scale * q with q in e4m3 and scale = 2^e, the smallest for which every |x| of the block's keys (or values) is at most 448 * 2^e.
In order, with i = 0..15 the token of the block and d the dim:
  keys    [i / 8][d / 16][i % 8][d % 16]     e4m3, 16*D bytes
  values  [d][i]                             e4m3, 16*D bytes
  scale of the keys, scale of the values, fp32, and 8 bytes that are 0
A scale is kept while tokens come to a block, or grows, and then what the block holds is rounded again; it starts anew when the
block's first token is written.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BLOCK = 16
MOST = 2.0 ** 100                            # larger magnitudes count as this
LEAST_EXP = -100                             # of a scale


# ---- cases -----------------------------------------------------------------------------------------------------------

def _tables(batch, page, table_pages, tokens, prompt, released, spare, **more):
    return dict(op="tables", batch=batch, page=page, table_pages=table_pages, tokens=tokens, prompt=prompt, released=released, spare=spare, **more)


def _rope(tokens, heads, kv_heads, head_dim, rotary, dtype, interleaved=False, inverse=False, scaled=False, far=131072, **more):
    return dict(op="rope", tokens=tokens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotary=rotary, dtype=dtype, interleaved=interleaved,
                inverse=inverse, scaled=scaled, far=far, **more)


def _append(tokens, kv_heads, head_dim, page, dtype, step, **more):
    return dict(op="append", tokens=tokens, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, step=step, **more)


def _attend(batch, length, kv_heads, group, head_dim, page, unit, queries=1, ragged=False, weights=False, dtype="bf16", keep=1.0, cap=0.0, slopes=False,
            window=0, sink=0, **more):
    return dict(op="attend", batch=batch, length=length, kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, unit=unit, queries=queries,
                ragged=ragged, weights=weights, dtype=dtype, keep=keep, cap=cap, slopes=slopes, window=window, sink=sink, **more)


def listed():
    return [
        # The tables of a decode step: 256 sequences, a token each, some of them finished, pages of 16 tokens: all launch and latency.
        _tables(256, 16, 2048, 256, 1, 0.02, 0.1, name="tables step"),
        # Prompts admitted together: 64 requests, 131072 new tokens at most, more asked for than there are pages.
        _tables(64, 32, 4096, 131072, 4000, 0.1, 0.25, name="tables prompts"),
        # Queries and keys of a decode step, one layer of an 8B-class model: 32 tokens.
        _rope(32, 32, 8, 128, 128, "bf16", name="rope step"),
        # The same of a prompt of full_8b's length, frequencies scaled for a long context: streaming.
        _rope(32768, 32, 8, 128, 128, "bf16", scaled=True, name="rope prompt"),
        # The gradient: turned back, pairs side by side, half of each head, fp32.
        _rope(4096, 16, 16, 128, 64, "fp32", interleaved=True, inverse=True, far=8192, name="rope gradient"),
        # One decode step of 32 sequences, one layer: a token each into blocks that hold others.
        _append(32, 8, 128, 16, "bf16", True, name="append step"),
        # The prompt of full_8b's length (2048 units of 16 tokens) written into the cache: streaming.
        _append(32768, 8, 128, 16, "bf16", False, name="append prompt"),
        # One sequence of about a thousand tokens, one layer: the smallest call of a decode loop.
        _attend(1, 1021, 8, 4, 128, 16, 16, weights=True, name="attend one"),
        # A decode batch of many lengths, an idle slot among them, scores capped.
        _attend(32, 8192, 8, 4, 128, 16, 16, ragged=True, cap=30.0, name="attend batch"),
        # One layer of long_70b: 4096 units of 32 tokens, eight queries a kv-head, the weight of every unit recorded.
        _attend(1, 131072, 8, 8, 128, 32, 32, weights=True, name="attend long"),
        # A window of 4096 tokens behind the first 64, a bias by distance, three drafted tokens verified with the last one, heads of 64, fp16.
        _attend(8, 32768, 8, 3, 64, 64, 1, queries=4, ragged=True, dtype="fp16", slopes=True, window=4096, sink=64, name="attend window"),
        # A chunk of 512 tokens of a prompt over the 32768 of full_8b's length.
        _attend(1, 32768, 8, 4, 128, 16, 16, queries=512, name="attend prompt"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rope", "rope", "append", "attend", "attend", "attend", "attend"])
    if op == "tables":
        batch, page = _log(rng, 1, 1024), rng.choice([16, 32, 48, 64])
        tokens = _log(rng, batch, 131072)
        return _tables(batch, page, _log(rng, 16, 4096 if batch <= 256 else 512), tokens, rng.choice([1, 1, 2, max(1, 2 * tokens // batch)]), rng.choice([0.0, 0.05, 0.3]),
                       rng.choice([0.02, 0.1, 0.5]))
    if op == "rope":
        heads, dim = rng.choice([1, 2, 5, 8, 16, 32]), rng.choice([32, 64, 96, 128, 256])
        kv = rng.choice([h for h in (1, 2, 5, 8) if heads % h == 0])
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        most = 32768 * 40 * 128 // ((heads + kv) * dim * (2 if dtype == "fp32" else 1))
        return _rope(_log(rng, 1, min(65536, most)), heads, kv, dim, rng.choice([dim, dim, dim // 2, dim // 4]), dtype, rng.random() < 0.4, rng.random() < 0.3,
                     rng.random() < 0.5, rng.choice([8192, 131072, 2 ** 24]))
    if op == "append":
        heads, dim, step = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 256]), rng.random() < 0.5
        most = 256 if step else min(32768, 32768 * 8 * 128 // (heads * dim))
        return _append(_log(rng, 1, most), heads, dim, rng.choice([16, 32, 64]), rng.choice(["bf16", "fp16", "fp32"]) if heads * dim <= 512 or step else
                       rng.choice(["bf16", "fp16"]), step)
    heads, dim, page, group = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 256]), rng.choice([16, 32, 64]), rng.randint(1, 8)
    length = _log(rng, 1, 131072)
    queries = rng.choice([1, 1, 1, 2, 3, _log(rng, 4, 512)])
    rows = 32768 * 512 * 8 * 4 // (length * heads * queries * group * max(1, dim // 128))
    batch = _log(rng, 1, max(1, min(64, rows, 4 * 131072 * 8 * 128 // (length * heads * dim * 2))))
    window = rng.choice([0, 0, 0, _log(rng, 1, 8192)])
    return _attend(batch, length, heads, group, dim, page, rng.choice([1, 2, 16, page]), queries if rows >= 1 else 1, rng.random() < 0.5, rng.random() < 0.5,
                   rng.choice(["bf16", "fp16"]), rng.choice([1.0, 1.0, 1.0, 0.4, 0.05]), rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3, window,
                   rng.choice([0, 4, 64]) if window else 0)


def _pages(case):
    return -(-case["length"] // case["page"])


def work(case):
    if case["op"] == "tables":
        n = min(case["tokens"], case["batch"] * case["prompt"])
        return {"bytes": 16 * case["tokens"] + 24 * case["batch"] + 8 * (n // case["page"] + case["batch"] // 8), "flops": 8 * case["tokens"]}
    if case["op"] == "rope":
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * case["head_dim"] * DTYPES[case["dtype"]].itemsize + 4 * case["tokens"], "flops": 3 * n * case["rotary"]}
    if case["op"] == "append":
        n, d, e = case["tokens"] * case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]].itemsize
        back = n * (BLOCK // 2 if case["step"] else 1)
        return {"bytes": 2 * n * d * e + n * 2 * d + back * 2 * d * (1 + e) + 16 * case["tokens"], "flops": 4 * n * d}
    b, h, g, d, t = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "queries"))
    length = case["length"] * (0.56 if case["ragged"] else 1.0)
    if case["window"]:
        length = min(length, case["window"] + case["sink"] + t - 1)
    seen = b * h * length * case["keep"]
    rows = b * t * h * g
    n = b * h * _pages(case) * case["page"] // case["unit"]
    return {"bytes": int(seen * (2 * d + 1) + rows * (4 * d + 4) + (4 * n if case["weights"] else 0) + (n / 8 if case["keep"] < 1 else 0) + 4 * b * _pages(case)),
            "flops": int(4 * seen * d * g * t)}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _rng(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(1_000_003 * (seed % 1_000_000_007) + 29)


def _keys_values(n, heads, dim, rng):
    """fp32 [n][heads][dim]: keys with a few strong channels a head and an offset, values without: as projections of a trained model have them."""
    strong = 1.0 + 3.0 * (torch.rand(heads, dim, generator=rng, device="cuda") > 0.95)
    offset = 0.5 * torch.randn(heads, dim, generator=rng, device="cuda") * strong
    k = torch.randn(n, heads, dim, generator=rng, device="cuda") * strong + offset
    return k, torch.randn(n, heads, dim, generator=rng, device="cuda"), strong


def _words(bits):
    """bool [..., U] -> int32 [..., ceil(U / 32)], bit u & 31 of word u >> 5."""
    u = bits.shape[-1]
    full = torch.nn.functional.pad(bits, (0, -u % 32)).view(*bits.shape[:-1], -1, 32).long()
    word = (full << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(word >= 2 ** 31, word - 2 ** 32, word).int()


def _slopes(heads):
    return torch.exp2(-8.0 * torch.arange(1, heads + 1, device="cuda") / heads)


def _frequencies(rotary, scaled):
    """Radians a token, float64; scaled: a ramp over the dims between frequencies as they are and divided by 8, and what the results are multiplied by."""
    half = rotary // 2
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    if not scaled:
        return f.cuda(), 1.0
    turns = f * 8192 / (2 * math.pi)
    ramp = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
    return (f * (ramp + (1.0 - ramp) / 8.0)).cuda(), 0.1 * math.log(8.0) + 1.0


def _prepare_tables(case, rng):
    b, page, width, tokens = case["batch"], case["page"], case["table_pages"], case["tokens"]
    most = width * page
    lens = (most * 0.9 * torch.rand(b, generator=rng, device="cuda") ** 2).long()
    if case["prompt"] > 1:                                      # a few of the requests have tokens already
        lens = torch.where(torch.rand(b, generator=rng, device="cuda") < 0.7, torch.zeros_like(lens), lens)
    used = (lens + page - 1) // page
    free = max(1, int(case["spare"] * max(b, b * case["prompt"] // page + 1)) if case["prompt"] == 1 else int(0.7 * tokens / page) + 1)
    pages = b * width + free                                    # the pool serves other batches too
    order = torch.randperm(pages, generator=rng, device="cuda").int()
    j = torch.arange(width, device="cuda")[None]
    held = j < used[:, None]
    rank = (held.view(-1).long().cumsum(0) - 1).view(b, width)
    table = torch.where(held, order[rank.clamp(min=0)], -1).int()
    head = int(torch.randint(0, pages, (1,), generator=rng, device="cuda"))
    ring = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(free, device="cuda")) % pages] = order[pages - free:]
    new = (case["prompt"] * (0.5 + torch.rand(b, generator=rng, device="cuda"))).long().clamp(min=1)
    x = torch.rand(b, generator=rng, device="cuda")
    new = torch.where(x < case["released"], -torch.ones_like(new), torch.where(x > 0.97, torch.zeros_like(new), new)).int()
    state = torch.tensor([head, free], dtype=torch.int32, device="cuda")
    return dict(case=case, new=new, lens=lens.int(), table=table, ring=ring, state=state)


def prepare(case, seed):
    rng = _rng(seed)
    if case["op"] == "tables":
        return _prepare_tables(case, rng)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "rope":
        n, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
        fused = torch.randn(n, (h + 2 * kv) * d, generator=rng, device="cuda").to(dtype)       # one projection's output; the values stay
        q, k = fused[:, : h * d].view(n, h, d), fused[:, h * d: (h + kv) * d].view(n, kv, d)
        if n <= 256:
            at = torch.randint(0, case["far"], (n,), generator=rng, device="cuda")
        else:
            at = torch.arange(n, device="cuda") + int(torch.randint(0, max(1, case["far"] - n), (1,), generator=rng, device="cuda"))
        f, factor = _frequencies(case["rotary"], case["scaled"])
        return dict(case=case, q=q, k=k, positions=at.int(), frequencies=f, factor=factor)
    h, d, page = case["kv_heads"], case["head_dim"], case["page"]
    size = page // BLOCK * (2 * BLOCK * d + 16)
    if case["op"] == "append":
        n = case["tokens"]
        k, v, _ = _keys_values(n, h, d, rng)
        used = -(-n // page)
        if case["step"]:                                        # a token of each sequence, somewhere in its last page
            pages = 2 * n + 3
            order = torch.randperm(pages, generator=rng, device="cuda")[:n]
            slots = order * page + torch.randint(0, page, (n,), generator=rng, device="cuda")
            kk, vv, _ = _keys_values(pages * page, h, d, rng)
            size_of = 0.7 + 0.6 * torch.rand(pages, 1, 1, 1, generator=rng, device="cuda")
            cache = _packed((kk.view(pages, page, h, d) * size_of).transpose(1, 2), (vv.view(pages, page, h, d) * size_of).transpose(1, 2))
            place = torch.arange(BLOCK, device="cuda")[None]
            back = torch.where(place <= slots[:, None] % BLOCK, slots[:, None] // BLOCK * BLOCK + place, -1).view(-1)
        else:
            pages = 2 * used + 3
            order = torch.randperm(pages, generator=rng, device="cuda")[:used]
            slots = (order[:, None] * page + torch.arange(page, device="cuda")).view(-1)[:n].contiguous()
            cache = torch.zeros(pages, h, size, dtype=torch.uint8, device="cuda")
            back = slots
        return dict(case=case, k=k.to(dtype), v=v.to(dtype), slots=slots.contiguous(), back=back.contiguous(), cache=cache)
    b, g, t, length, used = case["batch"], case["group"], case["queries"], case["length"], _pages(case)
    pages = b * used + 5
    table = torch.randperm(pages, generator=rng, device="cuda")[: b * used].view(b, used)
    cache = torch.zeros(pages, h, size, dtype=torch.uint8, device="cuda")
    q = torch.empty(b, t, h * g, d, dtype=dtype, device="cuda")
    for i in range(b):                                          # what earlier steps left in the cache
        k, v, strong = _keys_values(used * page, h, d, rng)
        cache[table[i]] = _packed(k.view(used, page, h, d).transpose(1, 2), v.view(used, page, h, d).transpose(1, 2))
        # scores with a standard deviation of about 2.5: a few units hold most of the weight
        q[i] = (2.5 * torch.randn(t, h, g, d, generator=rng, device="cuda") / strong[:, None]).reshape(t, h * g, d).to(dtype)
    lens = torch.full((b,), length, device="cuda")
    if case["ragged"]:
        lens = (length * (0.125 + 0.875 * torch.rand(b, generator=rng, device="cuda"))).long().clamp(1, length)
        lens[0] = length
        if b > 4:
            lens[-1] = 0                                        # an idle slot of the batch
    units = None
    if case["keep"] < 1.0:
        n = used * page // case["unit"]
        here = torch.arange(n, device="cuda")[None, None] * case["unit"] < lens[:, None, None]
        score = torch.rand(b, h, n, generator=rng, device="cuda").masked_fill(~here, -1.0)
        many = (case["keep"] * lens / case["unit"]).ceil().long()[:, None, None]
        units = _words(((score.argsort(-1, descending=True).argsort(-1) < many) & here).view(-1))
    return dict(case=case, q=q, cache=cache, table=table.int().contiguous(), lens=lens.int(), units=units, scale=d ** -0.5,
                slopes=_slopes(h * g) if case["slopes"] else None)


# ---- the operators ---------------------------------------------------------------------------------------------------

def _tables_plain(s):
    case, table, ring = s["case"], s["table"], s["ring"]
    page, (b, width), tokens, pages = case["page"], table.shape, case["tokens"], ring.numel()
    n, dev = s["new"].long(), table.device
    released = n < 0
    n = n.clamp(min=0)
    len0 = s["lens"].long().clamp(0, width * page)
    old = (len0 + page - 1) // page
    need = (len0 + n + page - 1) // page - old
    fits = ~released & (len0 + n <= width * page)
    head, count = s["state"].long().unbind()
    asked = torch.where(fits, need, 0).cumsum(0)
    total = torch.where(fits, n, 0).cumsum(0)
    yes = fits & ((need == 0) | (asked <= count)) & ((n == 0) | (total <= tokens))
    given, new = torch.where(yes, need, 0), torch.where(yes, n, 0)
    ends = new.cumsum(0)
    starts = torch.cat((torch.zeros_like(ends[:1]), ends))
    first = given.cumsum(0) - given
    at = torch.arange(tokens, device=dev)
    here = at < ends[-1]
    row = torch.searchsorted(ends, at, right=True).clamp(max=b - 1)
    pos = len0[row] + at - starts[row]
    j = (pos // page).clamp(0, width - 1)
    fresh = j >= old[row]
    got = torch.where(fresh, ring[(head + first[row] + j - old[row]) % pages].long(), table[row, j].long())
    good = here & (got >= 0) & (got < pages)
    slots = torch.where(good, got * page + pos % page, -1)
    flat = torch.cat((table.view(-1), table.new_zeros(1)))      # the last place takes what is written nowhere
    entry = torch.arange(width, device=dev)[None]
    back = released[:, None] & (entry < old[:, None]) & (table >= 0) & (table < pages)
    rank = back.view(-1).long().cumsum(0) - 1
    more = torch.cat((ring, ring.new_zeros(1)))
    more[torch.where(back.view(-1), (head + count + rank) % pages, pages)] = table.view(-1)
    flat[torch.where(here & fresh, row * width + j, b * width)] = got.int()
    table.copy_(flat[:-1].view(b, width))
    ring.copy_(more[:-1])
    state = torch.stack(((head + given.sum()) % pages, count - given.sum() + back.sum())).int()
    lens = torch.where(released, 0, len0 + new).int()
    return [slots, torch.where(here, pos, 0).int(), torch.where(here, row, -1).int(), starts.int(), (yes | released).int(), lens, state, table, ring]


def _rope_plain(s):
    case, f = s["case"], s["frequencies"]
    r = case["rotary"]
    angle = s["positions"].double()[:, None] * f[None]
    if case["inverse"]:
        angle = -angle
    cos, sin = (torch.cos(angle) * s["factor"]).float()[:, None], (torch.sin(angle) * s["factor"]).float()[:, None]
    out = []
    for x in (s["q"], s["k"]):
        y = x.float()
        part = y[..., :r]
        a, b = (part[..., 0::2], part[..., 1::2]) if case["interleaved"] else (part[..., : r // 2], part[..., r // 2:])
        a, b = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
        out.append(torch.cat((turned, y[..., r:]), -1).to(x.dtype))
    return out


def _exponent(most):
    """e of the smallest 2^e with most <= 448 * 2^e, as int32."""
    m, e = torch.frexp(most)
    return torch.where(m <= 0.875, e - 9, e - 8).clamp(min=LEAST_EXP)


def _power(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _e4m3(x):
    return x.to(torch.float8_e4m3fn)


def _cleaned(x):
    return torch.nan_to_num(x.float(), nan=0.0, posinf=MOST, neginf=-MOST).clamp(-MOST, MOST)


def _packed(k, v):
    """fp32 keys and values [pages][kv_heads][page][D] -> uint8 [pages][kv_heads][page bytes], the layout at the top of the file."""
    pages, h, page, d = k.shape
    parts, scales = [], []
    for x, is_key in ((k, True), (v, False)):
        x = _cleaned(x.reshape(pages, h, page // BLOCK, BLOCK, d))
        most = x.abs().amax((-1, -2))
        scale = torch.where(most > 0, _power(_exponent(most)), 0.0)
        q = _e4m3(x / torch.where(scale > 0, scale, 1.0)[..., None, None]).view(torch.uint8)
        q = q.view(*q.shape[:3], 2, 8, d // 16, 16).transpose(-3, -2) if is_key else q.transpose(-1, -2)
        parts.append(q.reshape(pages, h, page // BLOCK, -1))
        scales.append(scale)
    meta = torch.stack((*scales, torch.zeros_like(scales[0]), torch.zeros_like(scales[0])), -1).view(torch.uint8)
    return torch.cat((*parts, meta), -1).reshape(pages, h, -1)


def _held(blocks, d):
    """uint8 blocks [..., 32 * D + 16] -> e4m3 values as fp32 [..., 16, D] and scales [...] of the keys, the same of the values."""
    lead = blocks.shape[:-1]
    k, v, meta = blocks[..., : 16 * d], blocks[..., 16 * d: 32 * d], blocks[..., 32 * d: 32 * d + 8].contiguous().view(torch.float32)
    k = k.contiguous().view(torch.float8_e4m3fn).float().view(*lead, 2, d // 16, 8, 16).transpose(-3, -2).reshape(*lead, 16, d)
    v = v.contiguous().view(torch.float8_e4m3fn).float().view(*lead, d, 16).transpose(-1, -2)
    return (k, meta[..., 0]), (v, meta[..., 1])


def _append_plain(s):
    cache, slots, back = s["cache"], s["slots"], s["back"]
    pages, h, _ = cache.shape
    d, page = s["case"]["head_dim"], s["case"]["page"]
    per = page // BLOCK
    blocks = cache.view(pages, h, per, -1)
    many = pages * per                                          # blocks of a head; one more takes what is written nowhere
    where = torch.where((slots >= 0) & (slots < pages * page), slots // BLOCK, many)
    place = slots % BLOCK
    fresh = torch.zeros(many + 1, dtype=torch.bool, device=slots.device).index_fill_(0, torch.where(place == 0, where, many), True)
    new, scales = [], []
    for x, (q, scale) in zip((s["k"], s["v"]), _held(blocks, d)):
        x = _cleaned(x)
        most = torch.zeros(many + 1, h, device=x.device).index_reduce_(0, where, x.abs().amax(-1), "amax")[:-1]
        old = scale.transpose(1, 2).reshape(many, h)
        old = torch.where(fresh[:-1, None], 0.0, old)
        now = torch.maximum(old, torch.where(most > 0, _power(_exponent(most)), 0.0))
        unit = torch.where(now > 0, now, 1.0)
        grown = (old / unit).view(pages, per, h).transpose(1, 2)
        q = torch.where((now > old).view(pages, per, h).transpose(1, 2)[..., None, None], _e4m3(q * grown[..., None, None]).float(), q)
        q = torch.cat((q.permute(0, 2, 3, 1, 4).reshape(many, BLOCK, h, d), q.new_zeros(1, BLOCK, h, d)))
        unit = torch.cat((unit, unit.new_ones(1, h)))
        q[where, place] = _e4m3(x / unit[where][..., None]).float()
        new.append(_e4m3(q[:-1]).view(torch.uint8).view(pages, per, BLOCK, h, d).permute(0, 3, 1, 2, 4))
        scales.append(now.view(pages, per, h).transpose(1, 2))
    k = new[0].reshape(pages, h, per, 2, 8, d // 16, 16).transpose(-3, -2).reshape(pages, h, per, -1)
    v = new[1].transpose(-1, -2).reshape(pages, h, per, -1)
    zero = torch.zeros_like(scales[0])
    meta = torch.stack((scales[0], scales[1], zero, zero), -1).contiguous().view(torch.uint8)
    touched = torch.zeros(many + 1, dtype=torch.bool, device=slots.device).index_fill_(0, where, True)[:-1].view(pages, 1, per, 1)
    blocks.copy_(torch.where(touched, torch.cat((k, v, meta), -1), blocks))
    there = (back >= 0) & (back < pages * page)
    at = torch.where(there, back, 0)
    found = blocks[at // page, :, at % page // BLOCK]                           # [T][H][bytes]
    out = []
    for q, scale in _held(found, d):
        x = q[torch.arange(len(at), device=at.device), :, at % BLOCK] * scale[..., None]
        out.append(torch.where(there[:, None, None], x, 0.0).to(s["k"].dtype))
    return out


def _seen(case, lens, many, units, kv_heads):
    """Truth [B][1 or H][T][1][tokens]: what each query sees."""
    t, dev = case["queries"], lens.device
    at = lens[:, None] - t + torch.arange(t, device=dev)                        # positions of the queries
    i = torch.arange(many, device=dev)
    seen = i <= at[:, :, None]
    if case["window"]:
        seen = seen & ((i > at[:, :, None] - case["window"]) | (i < case["sink"]))
    seen = seen[:, None, :, None, :]
    if units is not None:
        u = torch.arange(len(lens) * kv_heads * (many // case["unit"]), device=dev)
        bits = (units[u >> 5].long() >> (u & 31)) & 1
        seen = seen & bits.bool().view(len(lens), kv_heads, -1).repeat_interleave(case["unit"], -1)[:, :, None, None, :]
    return seen, at


def _attend_plain(s):
    case, q, lens = s["case"], s["q"], s["lens"].long()
    b, h, g, d, t = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "queries"))
    blocks = s["cache"][s["table"].long()].transpose(1, 2).reshape(b, h, -1, 32 * d + 16)
    k, v = ((x * scale[..., None, None]).reshape(b, h, -1, d) for x, scale in _held(blocks, d))
    many, unit = k.shape[2], case["unit"]
    seen, at = _seen(case, lens, many, s["units"], h)
    x = q.float().view(b, t, h, g, d).permute(0, 2, 1, 3, 4).reshape(b, h, t * g, d)
    score = (torch.matmul(x, k.transpose(-1, -2)) * s["scale"]).view(b, h, t, g, many)
    if case["cap"]:
        score = torch.tanh(score / case["cap"]) * case["cap"]
    if s["slopes"] is not None:
        far = torch.arange(many, device=q.device) - at[:, None, :, None, None]
        score = score + s["slopes"].view(1, h, 1, g, 1) * far
    score = score.masked_fill(~seen, -math.inf)
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


def run(s):
    case = s["case"]
    if own:
        from paper_2508_13231_b200 import kvp
        if case["op"] == "tables":
            r = kvp.block_tables(s["new"], s["lens"], s["table"], s["ring"], s["state"], case["page"], case["tokens"])
            return [r["slots"], r["positions"], r["rows"], r["starts"], r["granted"], r["lens"], r["state"], s["table"], s["ring"]]
        if case["op"] == "rope":
            return list(kvp.rope(s["q"], s["k"], s["positions"], s["frequencies"], interleaved=case["interleaved"], inverse=case["inverse"],
                                 scale=s["factor"]))
        if case["op"] == "append":
            kvp.cache8_append(s["cache"], s["k"], s["v"], s["slots"])
            return list(kvp.cache8_read(s["cache"], s["back"], case["head_dim"], s["k"].dtype))
        r = kvp.attend8(s["q"], s["cache"], s["table"], s["lens"], unit_tokens=case["unit"], scale=s["scale"], units=s["units"], cap=case["cap"],
                        slopes=s["slopes"], window=case["window"], sink=case["sink"], want_lse=True, want_weights=case["weights"])
        return [r["out"], r["lse"]] + ([r["weights"]] if case["weights"] else [])
    if case["op"] == "tables":
        return _tables_plain(s)
    if case["op"] == "rope":
        return _rope_plain(s)
    return _append_plain(s) if case["op"] == "append" else _attend_plain(s)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _values(code):
    """uint8 e4m3 codes -> what they stand for, in 64 bits."""
    sign, e, m = 1.0 - 2.0 * (code >> 7).double(), ((code >> 3) & 15).double(), (code & 7).double()
    return sign * torch.where(e > 0, (8 + m) * torch.exp2(e - 10), m * 2.0 ** -9)


def _nearest(x):
    """x (64 bits, at most 448) rounded to e4m3: three bits behind the first, whole multiples of 2^-9 at least; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _block_values(cache, d, block, head, is_key):
    """The 16 tokens of the blocks (numbers over all pages) of one head: e4m3 values [n][16][D] and scales [n], in 64 bits."""
    per = cache.shape[2] // (32 * d + 16)
    raw = cache[block // per, head].view(len(block), per, -1)[torch.arange(len(block), device=cache.device), block % per]
    i, dim = torch.arange(16, device=cache.device)[:, None], torch.arange(d, device=cache.device)[None]
    where = ((i // 8) * (d // 16) + dim // 16) * 128 + (i % 8) * 16 + dim % 16 if is_key else 16 * d + dim * 16 + i
    first = 32 * d + (0 if is_key else 4)
    return _values(raw[:, where].long()), raw[:, first: first + 4].contiguous().view(torch.float32)[:, 0].double()


def _exact_append(s):
    case, slots, back = s["case"], s["slots"], s["back"]
    d, h = case["head_dim"], case["kv_heads"]
    block, place = slots // BLOCK, slots % BLOCK
    which, inverse = torch.unique(block, return_inverse=True)
    fresh = torch.zeros(len(which), dtype=torch.bool, device=block.device)
    fresh[inverse[place == 0]] = True
    out = []
    for x, is_key in ((s["k"], True), (s["v"], False)):
        found = torch.zeros(len(back), h, d, dtype=torch.float64, device=x.device)
        for head in range(h):
            y = x[:, head].double()
            most = torch.zeros(len(which), dtype=torch.float64, device=x.device).scatter_reduce_(0, inverse, y.abs().amax(-1), "amax")
            e = torch.ceil(torch.log2(most.clamp(min=1e-30) / 448.0))
            e = torch.where(448.0 * torch.exp2(e - 1) >= most, e - 1, torch.where(448.0 * torch.exp2(e) < most, e + 1, e))
            held, old = _block_values(s["cache"], d, which, head, is_key)
            old = torch.where(fresh, 0.0, old)
            scale = torch.maximum(torch.where(most > 0, torch.exp2(e), 0.0), old)
            unit = torch.where(scale > 0, scale, 1.0)
            held = torch.where((scale > old)[:, None, None], _nearest(held * (old / unit)[:, None, None]), held)
            held[inverse, place] = _nearest(y / unit[inverse][:, None])
            there = back >= 0
            at = torch.searchsorted(which, back[there] // BLOCK)
            found[there, head] = (held * scale[:, None, None])[at, back[there] % BLOCK]
        out.append(found)
    return out


def _exact_rope(s):
    case, r = s["case"], s["case"]["rotary"]
    at = s["positions"].double()[:, None] * s["frequencies"][None]
    turn = torch.polar(torch.full_like(at, s["factor"]), -at if case["inverse"] else at)[:, None]
    out = []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return out


def exact(case, seed):
    if case["op"] == "tables":
        return None                                             # whole numbers: they have to be equal
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "rope":
        return _exact_rope(s)
    b, h, g, d, t, unit = (case[k] for k in ("batch", "kv_heads", "group", "head_dim", "queries", "unit"))
    many = _pages(case) * case["page"]
    n = many // unit
    out = torch.zeros(b, t, h * g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, t, h * g), -math.inf, dtype=torch.float64, device="cuda")
    got = torch.zeros(b, h, n, dtype=torch.float64, device="cuda")
    per = case["page"] // BLOCK
    step = max(1, min(t, 2 ** 28 // (many * g)))                # queries at a time
    for i in range(b):
        length = int(s["lens"][i])
        if not length:
            continue
        block = (s["table"][i].long()[:, None] * per + torch.arange(per, device="cuda")).view(-1)
        seen, at = _seen(dict(case, batch=1), s["lens"][i: i + 1].long(), many, None, h)
        seen, at = seen[0, 0, :, 0], at[0]
        for j in range(h):
            k, v = (x.mul(scale[:, None, None]).view(-1, d) for x, scale in (_block_values(s["cache"], d, block, j, key) for key in (True, False)))
            keep = torch.ones(many, dtype=torch.bool, device="cuda")
            if s["units"] is not None:
                u = (i * h + j) * n + torch.arange(many, device="cuda") // unit
                keep = ((s["units"][u >> 5].long() >> (u & 31)) & 1) > 0
            for r in range(0, t, step):
                rows = slice(r, min(t, r + step))
                x = torch.einsum("tgd,md->tgm", s["q"][i, rows, j * g: (j + 1) * g].double(), k) * s["scale"]
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if s["slopes"] is not None:
                    x = x + s["slopes"][j * g: (j + 1) * g].double()[None, :, None] * (torch.arange(many, device="cuda") - at[rows, None])[:, None]
                ok = (seen[rows] & keep)[:, None]
                x = x.masked_fill(~ok, -math.inf)
                lse[i, rows, j * g: (j + 1) * g] = torch.logsumexp(x, -1)
                p = torch.where(ok, torch.exp(x - lse[i, rows, j * g: (j + 1) * g, None]), 0.0)
                out[i, rows, j * g: (j + 1) * g] = p @ v
                got[i, j].index_add_(0, torch.arange(many, device="cuda") // unit, p.sum((0, 1)))
    return [out, lse] + ([got] if case["weights"] else [])
