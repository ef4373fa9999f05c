"""Synthetic reruns of the paper's sensitivity study (Section IV-B, Fig. 3-5) on one B200.

    python -m paper_2508_13231_b200.figures [--quick] [--recorded [--bits 8]]

One attention head at token granularity: 4096 tokens (512 B of K+V each), 512 decode steps, HBM room for 25% of
them, 8 TB/s HBM against 0.9 TB/s off-package, Zipf(1.1) importance with AR(1) drift. The recorded LLaMA-3.1-8B /
LongBench traces of the paper are not available; these traces are synthetic, so the numbers show the same trends,
not the paper's values. Strategies (Section IV-A): Unlimited HBM, Static Placement (first come), Reactive (LRU),
Page granularity (16 tokens), SA-guided = the paper's annealer over the look-ahead policy's (W, R), followed by
direct annealing of the schedule it found. Everything runs in the library's kernels; this file only calls them.

--recorded: the strategies on a trace of recorded attention weights, as the paper's are (Section IV-A): random keys, values and drifting queries
stand in for a model, tokens are decoded with attention over a cache held in 4 bits (the paper records a model with an unquantised one, so
these weights contain the error of 4 bits), and each step reads the units that received most weight. Beside them the placement by accumulated
weight, and what eviction by it leaves of the attention weight: the units evicted after a step are gone for all later ones.
--bits 8 records with a cache held in 8 bits (normal values are off by 0.027 of their deviation where 4 bits leave 0.078), with rotary positions and
with pages, slots and positions from the device's block tables.
"""
import argparse

import numpy as np
import torch

from . import kvp, workloads as wl

TOKENS, STEPS, CAP, BPU = 4096, 512, 1024, 512
BW = (8 * wl.TB, 9 * wl.TB // 10, 9 * wl.TB // 10)


def strategies(topk, rho, quick=False, seed=0):
    """-> dict name -> (total ticks, HBM hit rate)."""
    tp = wl.custom_trace_params(1, TOKENS, STEPS, topk, rho, zipf=(1.1, 1.1), seed=seed)
    base = torch.from_numpy(tp["base"]).cuda()
    A = kvp.trace_generate(**{k: v for k, v in tp.items() if k != "base"}, base=base)
    prob = kvp.Problem(TOKENS, BPU, STEPS, A, CAP, *BW)
    unlimited = kvp.Problem(TOKENS, BPU, STEPS, A, TOKENS, *BW)
    accessed = STEPS * topk

    def score(p, sched):
        ticks = int(p.eval(sched, want_steps=False, want_seconds=False)["total_ticks"][0])
        hits = int(p.eval_counts(sched)[0, :, 0].sum())
        return ticks, hits / accessed

    out = {}
    ones = torch.full((STEPS, TOKENS // 32), -1, dtype=torch.int32, device="cuda")
    out["unlimited"] = score(unlimited, ones)
    static = prob.policy_lookahead([1], [0])[0].contiguous()              # R = 0: first-come placement, no migration
    out["static"] = score(prob, static)
    out["reactive"] = score(prob, prob.policy_reactive())
    out["page16"] = score(prob, prob.policy_page(16))
    w_max = 16 if quick else 64
    table = prob.wr_grid(w_max, 11)
    _, best = kvp.wr_anneal(table, kvp.wr_params(chains=64, iters=2000, seed=seed, levels=32, early_stop_permille=1))
    look = prob.policy_lookahead([best.best_w], [100 * best.best_r])[0].contiguous()
    out["lookahead_sa"] = score(prob, look) + ((best.best_w, best.best_r / 10),)
    prm = prob.make_params(chains=64 if quick else 256, moves=50_000 if quick else 400_000, seed=seed, p0=1e-3,
                           init_mode=kvp.INIT_USER, init_schedule=look)
    res = prob.anneal(prm)
    out["sa_guided"] = score(prob, res["best_schedule"])
    prob.close(); unlimited.close()
    return out


def record8(cfg, seed=0):
    """record() with a cache held in 8 bits, rotary positions and the device's block tables."""
    h, d, page = cfg["kv_heads"], cfg["head_dim"], cfg["unit_tokens"]
    total = cfg["prompt"] + cfg["steps"]
    n = -(-total // page)
    rng = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *size: torch.randn(*size, generator=rng, device="cuda")  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = torch.zeros(n, h, kvp.cache8_page_bytes(d, page), dtype=torch.uint8, device="cuda")
    table, lens, state = torch.full((1, n), -1, dtype=torch.int32, device="cuda"), i32(0), i32(0, n)
    ring = torch.randperm(n, generator=rng, device="cuda").int()
    frequencies, scale = kvp.rope_frequencies(d, scaling="ramp", factor=4.0)
    frequencies = frequencies.cuda()

    def append(q, k, v):
        """The next tokens: their pages and slots, rotary positions of queries and keys, keys and values into the cache -> the queries."""
        r = kvp.block_tables(i32(len(q)), lens, table, ring, state, page, len(q), lens_out=lens, state_out=state)
        q, k = kvp.rope(q, k, r["positions"], frequencies, scale=scale)
        kvp.cache8_append(cache, k, v, r["slots"])
        return q

    k, v, q = rand(total, h, d).bfloat16(), rand(total, h, d).bfloat16(), rand(cfg["queries"], d)
    p = cfg["prompt"]
    append(q.bfloat16().expand(p, -1, -1), k[:p], v[:p])
    weights = torch.empty(cfg["steps"], h * n, device="cuda")
    for s in range(cfg["steps"]):
        q = cfg["rho"] * q + (1 - cfg["rho"] ** 2) ** 0.5 * rand(*q.shape)
        turned = append((2.5 * q).bfloat16()[None], k[p + s: p + s + 1], v[p + s: p + s + 1])
        kvp.attend8(turned, cache, table, lens, weights=weights[s])
    return weights, n


def record(cfg, seed=0):
    """Decodes cfg["steps"] tokens of one layer -> weights [steps][kv_heads * units] (kvp.attend), units per kv-head."""
    h, d, page = cfg["kv_heads"], cfg["head_dim"], cfg["unit_tokens"]
    total = cfg["prompt"] + cfg["steps"]
    n = -(-total // page)
    rng = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *size: torch.randn(*size, generator=rng, device="cuda")  # noqa: E731
    cache = torch.zeros(n, h, kvp.cache_page_bytes(d, page), dtype=torch.uint8, device="cuda")
    table = torch.randperm(n, generator=rng, device="cuda").int()[None]
    slots = table[0].long().repeat_interleave(page)[:total] * page + torch.arange(total, device="cuda") % page
    k, v, q = rand(total, h, d).bfloat16(), rand(total, h, d).bfloat16(), rand(cfg["queries"], d)
    kvp.cache_append(cache, k[:cfg["prompt"]], v[:cfg["prompt"]], slots[:cfg["prompt"]])
    weights = torch.empty(cfg["steps"], h * n, device="cuda")
    for s in range(cfg["steps"]):
        t = cfg["prompt"] + s
        kvp.cache_append(cache, k[t:t + 1], v[t:t + 1], slots[t:t + 1])
        q = cfg["rho"] * q + (1 - cfg["rho"] ** 2) ** 0.5 * rand(*q.shape)
        kvp.attend((2.5 * q).bfloat16()[None], cache, table, torch.tensor([t + 1], dtype=torch.int32, device="cuda"), weights=weights[s])
    return weights, n


def weight_kept(weights, cfg, n, share):
    """Eviction to `share` of a head's units after every step -> share of the next steps' attention weight on the units kept."""
    h = cfg["kv_heads"]
    tokens = cfg["prompt"] + 1 + torch.arange(cfg["steps"], device="cuda")
    exist = ((tokens + cfg["unit_tokens"] - 1) // cfg["unit_tokens"]).int()[:, None].expand(-1, h).contiguous()
    rows = kvp.evict(weights, h, max(4, int(share * n)), sink=1, recent=2, exist=exist, carry=True)["kept"]
    bits = torch.from_numpy(wl.unpack_bits(rows.cpu().numpy().view(np.uint32), h * n)).cuda()
    return float((weights[1:] * bits[:-1]).sum() / weights[1:].sum())


def recorded(name, quick=False, seed=0, bits=4):
    """-> dict strategy -> (total ticks, HBM hit rate), dict share of the units kept -> share of the attention weight they receive."""
    cfg = wl.RECORDED[name]
    h, steps = cfg["kv_heads"], cfg["steps"]
    weights, n = record8(cfg, seed) if bits == 8 else record(cfg, seed)
    access = kvp.trace_weights(weights, h, cfg["topk"])
    units, cap = h * n, int(cfg["share"] * h * n)
    page_bytes = kvp.cache8_page_bytes if bits == 8 else kvp.cache_page_bytes
    prob = kvp.Problem(units, page_bytes(cfg["head_dim"], cfg["unit_tokens"]), steps, access, cap, *cfg["bw"])

    def score(sched):
        counts = prob.eval_counts(sched)[0].long().sum(0)
        return int(prob.eval(sched, want_steps=False, want_seconds=False)["total_ticks"][0]), int(counts[0]) / accessed

    accessed = int(np.unpackbits(access.cpu().numpy().view(np.uint8)).sum())
    out = {"static": score(prob.policy_lookahead([1], [0])[0].contiguous()), "reactive": score(prob.policy_reactive())}
    held = prob.policy_accumulated(weights, h, sink=1, decay_q=61440)
    out["accumulated"] = score(held)
    res = prob.anneal(prob.make_params(chains=64 if quick else 256, moves=20_000 if quick else 200_000, seed=seed, p0=1e-3,
                                       init_mode=kvp.INIT_USER, init_schedule=held))
    out["sa_guided"] = score(res["best_schedule"])
    prob.close()
    return out, {share: weight_kept(weights, cfg, n, share) for share in (0.5, 0.25, 0.125)}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--quick", action="store_true")
    ap.add_argument("--recorded", action="store_true")
    ap.add_argument("--bits", type=int, choices=(4, 8), default=4, help="of the cache that --recorded decodes with")
    args = ap.parse_args()
    if args.recorded:
        name = "recorded_small" if args.quick else "recorded_8b"
        out, kept = recorded(name, args.quick, bits=args.bits)
        print(f"Recorded attention weights ({name}, cache in {args.bits} bits): tokens/s normalised to Static Placement, HBM hit rate\n")
        print("| " + " | ".join(out) + " |\n|" + "---|" * len(out))
        print("| " + " | ".join(f"{out['static'][0] / t:.2f}, {r:.3f}" for t, r in out.values()) + " |\n")
        print("Eviction by accumulated weight: share of the later steps' attention weight on the units kept\n")
        print("| " + " | ".join(f"{s:.3f} of the units" for s in kept) + " |\n|" + "---|" * len(kept))
        print("| " + " | ".join(f"{w:.3f}" for w in kept.values()) + " |")
        return
    names = ["unlimited", "static", "reactive", "page16", "lookahead_sa", "sa_guided"]
    print("Fig. 3 analogue: tokens/s normalised to Static Placement (rho = 0.95)\n")
    print("| sparsity | " + " | ".join(names) + " | best (W, R) |")
    print("|---|" + "---|" * (len(names) + 1))
    keep = {}
    for sparsity in (50, 60, 70, 80, 90, 95):
        topk = TOKENS * (100 - sparsity) // 100
        r = strategies(topk, 0.95, args.quick)
        keep[sparsity] = r
        print(f"| {sparsity}% | " + " | ".join(f"{r['static'][0] / r[n][0]:.2f}" for n in names) +
              f" | {r['lookahead_sa'][2]} |")
    print("\nFig. 4 analogue: tokens/s normalised to Unlimited HBM at 60% sparsity\n")
    print("| variation | " + " | ".join(names[1:]) + " |")
    print("|---|" + "---|" * (len(names) - 1))
    for label, rho in (("low (rho 0.99)", 0.99), ("high (rho 0.5)", 0.5)):
        r = strategies(TOKENS * 40 // 100, rho, args.quick)
        print(f"| {label} | " + " | ".join(f"{r['unlimited'][0] / r[n][0]:.2f}" for n in names[1:]) + " |")
    print("\nFig. 5 analogue: HBM hit rate at 60% sparsity (rho = 0.95)\n")
    r = keep[60]
    print("| " + " | ".join(names[1:]) + " |")
    print("|" + "---|" * (len(names) - 1))
    print("| " + " | ".join(f"{r[n][1]:.3f}" for n in names[1:]) + " |")


if __name__ == "__main__":
    main()
