"""The attention operators that are timed on this framework: what a program that serves a graph transformer has them do.

Three kinds of work, each through the public calls of ``paper_2503_01281_amd``:

  attend  rows of a block attend over their lists of sources.  ``slots`` > 0: keys and values come from the 8-bit cache
          (``dci_attn_cached``), where a list entry names a source of the batch and ``slot_of`` that source's slot (-1: it has
          none and is left out); ``accumulate`` adds every slot's attention weight to the cache's counters.  ``slots`` = 0: keys
          and values are dense rows of the batch (``dci_attn_forward``), as in a model's later layers.
  store   rows are written into the 8-bit cache (``dci_kv_write``) and the blocks that they touch are read back
          (``dci_kv_read``), as for a layer that wants dense rows.
  admit   the nodes of a batch are looked up in the cache, and those without a slot get the slots of least accumulated
          weight (``dci_kv_admit``).

Keys, queries and values are N(0, 1) with a few wide columns, as projections have them; weights are log-normal; lists are those of a
power-law graph, with a preference for few sources.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = 2.0 ** -32  # of an accumulated weight
E_MIN, E_MAX = -100, 119  # exponents of the scales


def _attend(name, rows, mean, longest, sources, heads, dim, dtype, **kw):
    c = dict(name=name, op="attend", rows=rows, bound=rows, mean=mean, longest=longest, sources=sources, heads=heads, kv_heads=heads,
             dim=dim, dtype=dtype, slots=0, block=16, bias=0, accumulate=False, missing=0.0)
    c.update(kw)
    return c


def _store(name, rows, slots, heads, dim, dtype, block):
    return dict(name=name, op="store", rows=rows, slots=slots, kv_heads=heads, dim=dim, dtype=dtype, block=block)


def _admit(name, batch, nodes, slots, cached, repeats=0):
    return dict(name=name, op="admit", batch=batch, nodes=nodes, slots=slots, cached=cached, repeats=repeats)


def listed():
    return [
        # a single request: one node, the list of one hop; latency is all that counts
        _attend("one node", 1, 15.0, 15, 16, 4, 64, "fp32", slots=16_384),
        # input layer of a batch of 4,096 seeds at fan-outs 5, 10, 15 on a graph of products, hidden width 256; sized by its
        # bound, as the batch's sizes stay on the GPU; the weights are accumulated for later evictions
        _attend("input layer", 98_304, 12.0, 15, 400_000, 4, 64, "bf16", bound=131_072, slots=1_048_576, accumulate=True, missing=0.02),
        # the same with hidden width 128, in 32 bits, a bias on every edge
        _attend("input layer, edge bias", 67_584, 10.0, 15, 230_000, 4, 32, "fp32", slots=500_000, block=32, bias=1),
        # nothing divides anything: odd head width and count, some rows empty, some entries masked, single-slot scales
        _attend("odd widths", 10_007, 20.0, 64, 40_009, 3, 41, "fp16", slots=65_537, block=1, bias=3, missing=0.1, accumulate=True),
        # whole neighbour lists of hubs, shared key heads
        _attend("whole lists", 200, 5_000.0, 0, 500_000, 16, 64, "bf16", kv_heads=4, slots=524_288, block=64),
        # few rows with very long lists and wide heads: the largest
        _attend("long lists", 16, 40_000.0, 0, 600_000, 32, 128, "bf16", kv_heads=8, slots=655_360),
        # later layers: rows of the batch
        _attend("second layer", 24_576, 9.0, 10, 200_000, 4, 64, "fp32", bound=30_000),
        _attend("last layer, bf16", 4_096, 20.0, 25, 60_000, 8, 32, "bf16"),
        # the cache is filled in bulk; a batch's new rows go to scattered slots
        _store("bulk fill", 500_000, 500_000, 4, 64, "bf16", 16),
        _store("new rows", 20_011, 262_144, 4, 64, "fp32", 16),
        # a batch of 4,096 seeds, a request of a few
        _admit("admit a batch", 400_000, 2_449_029, 1_048_576, 0.4),
        _admit("admit a request", 3_000, 232_965, 65_536, 0.7, repeats=5),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend"] * 4 + ["store", "admit"])
    if op == "admit":
        slots = log_int(500, 1_000_000)
        batch = log_int(1, min(400_000, 2 * slots))
        return dict(op=op, batch=batch, nodes=max(slots + batch, log_int(20_000, 2_400_000)), slots=slots,
                    cached=round(rng.uniform(0.0, 0.95), 2), repeats=rng.choice([0, 0, batch // 7]))
    dim = rng.choice([16, 32, 64, 64, 128, rng.randint(1, 130)])
    kv = rng.randint(1, max(1, min(8, 512 // dim)))
    dtype = rng.choice(list(TYPES))
    block = rng.choice([1, 2, 4, 8, 16, 16, 32, 64])
    if op == "store":
        slots = log_int(64, 400_000)
        return dict(op=op, rows=slots if rng.random() < 0.4 else log_int(1, slots), slots=slots, kv_heads=kv, dim=dim, dtype=dtype,
                    block=block)
    cached = rng.random() < 0.7
    long = rng.random() < 0.3
    edges = 1_000_000 * 64 // max(64, kv * dim // 4)
    if long:
        rows = log_int(1, 300)
        mean, longest = float(log_int(100, max(101, min(40_000, edges // rows)))), 0
        group = rng.choice([1, 2, 4, 8])
    else:
        longest = rng.choice([2, 5, 8, 10, 15, 25, 64])
        mean = round(longest * rng.uniform(0.4, 1.0), 1)
        rows = log_int(1, max(2, min(100_000, int(edges / mean))))
        group = rng.choice([1, 1, 1, 2])
    sources = log_int(max(2, int(rows * mean / 20)), max(100, min(500_000, int(rows * mean))))
    return dict(op=op, rows=rows, bound=rows + rng.choice([0, rows // 3]), mean=mean, longest=longest, sources=sources,
                heads=kv * group, kv_heads=kv, dim=dim, dtype=dtype, slots=sources + log_int(1, 300_000) if cached else 0, block=block,
                bias=rng.choice([0, 0, 1, kv * group]), accumulate=cached and rng.random() < 0.4,
                missing=rng.choice([0.0, 0.1]) if cached else 0.0)


# ---- inputs --------------------------------------------------------------------------------------


def _width(dim):
    """Columns of a cached row's head: the head width on whole 16 bytes."""
    return (dim + 15) // 16 * 16


def _rows(n, heads, dim, dtype, gen):
    wide = 1.0 + 3.0 * (torch.rand(heads, dim, generator=gen, device="cuda") < 0.05)
    x = torch.randn(n, heads, dim, generator=gen, device="cuda") * wide
    return x.to(TYPES[dtype])


def _held(x):
    """e4m3 codes of x: the bytes that stand for the nearest values."""
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _cache_arrays(slots, heads, dim, block, gen):
    """(codes, scales) of a cache of N(0, 1) rows: codes [slots, 2, heads, width], scales [blocks, heads, 2]."""
    blocks, width = -(-slots // block), _width(dim)
    codes = torch.zeros(blocks * block, 2, heads, width, dtype=torch.uint8, device="cuda")
    scales = torch.empty(blocks, heads, 2, device="cuda")
    step = max(1, (1 << 27) // (block * heads * dim))
    for lo in range(0, blocks, step):
        hi = min(blocks, lo + step)
        x = torch.randn((hi - lo), block, 2, heads, dim, generator=gen, device="cuda")
        e = _exponent(x.abs().amax((1, 4)))
        scales[lo:hi] = torch.exp2(e).mT
        codes[lo * block:hi * block, ..., :dim] = _held(x * torch.exp2(-e)[:, None, :, :, None]).flatten(0, 1)
    return codes[:slots].contiguous(), scales


def _lists(case, gen):
    """indptr, src of rows * mean entries or so: lengths of sampled lists (at most `longest`), or log-normal ones."""
    n, mean, longest = case["rows"], case["mean"], case["longest"]
    z = torch.randn(n, generator=gen, device="cuda")
    if longest:
        share = mean / longest
        length = torch.where(z < -1.6, torch.zeros_like(z), (longest * (share + 0.6 * (z + 0.5))).round()).clamp(0, longest)
        if n < 8:
            length.fill_(mean)
    else:
        length = (mean * torch.exp(0.8 * z - 0.32)).round().clamp(0, 8 * mean)
        length = length * (mean * n / length.sum().clamp(min=1)).clamp(max=1)
        if n > 10:
            length[n // 3] = 0
    length = length.long()
    indptr = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    indptr[1:] = length.cumsum(0)
    e = int(indptr[-1])
    src = (case["sources"] * torch.rand(e, generator=gen, device="cuda", dtype=torch.float64) ** 2).int().clamp(max=case["sources"] - 1)
    return indptr, src


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"attend": _prepare_attend, "store": _prepare_store, "admit": _prepare_admit}[case["op"]](case, gen)
    s["case"] = case
    if own:
        import paper_2503_01281_amd as dci
        s["dci"], s["ctx"] = dci, dci.Context(0, stream=torch.cuda.current_stream())
        if case.get("slots"):
            s["cache"] = dci.KvCache.from_arrays(s["codes"], s["scales"], s["weight"].clone(), s["node"].clone(), case.get("dim", 16),
                                                 case.get("block", 16))
    torch.cuda.synchronize()
    return s


def _prepare_attend(case, gen):
    indptr, src = _lists(case, gen)
    heads, dim, bound, n = case["heads"], case["dim"], case["bound"], case["rows"]
    if bound > n:  # the arrays have the bound's size, the number of rows stays on the GPU
        indptr = torch.cat([indptr, torch.zeros(bound - n, dtype=torch.int64, device="cuda")])
    s = dict(indptr=indptr, src=src, q=_rows(bound, heads, dim, case["dtype"], gen), scale=1.0 / math.sqrt(dim), bias=None,
             n_dev=torch.tensor([n], dtype=torch.int64, device="cuda") if bound > n else None)
    if case["bias"]:
        s["bias"] = torch.randn(src.numel(), case["bias"], generator=gen, device="cuda")
        s["bias"][torch.rand(src.numel(), case["bias"], generator=gen, device="cuda") < 0.05] = -math.inf
    if case["slots"]:
        s["codes"], s["scales"] = _cache_arrays(case["slots"], case["kv_heads"], dim, case["block"], gen)
        slot_of = torch.randperm(case["slots"], generator=gen, device="cuda")[:case["sources"]].int()
        slot_of[torch.rand(slot_of.numel(), generator=gen, device="cuda") < case["missing"]] = -1
        s["slot_of"] = slot_of
        s["weight"] = (torch.rand(case["slots"], generator=gen, device="cuda") * 2.0 ** 33).long() + 1
        s["node"] = torch.arange(case["slots"], device="cuda")
    else:
        s["k"], s["v"] = (_rows(case["sources"], case["kv_heads"], dim, case["dtype"], gen) for _ in range(2))
    s["out"] = torch.zeros(bound, heads, dim, dtype=TYPES[case["dtype"]], device="cuda")
    s["lse"] = torch.zeros(bound, heads, device="cuda")
    return s


def _prepare_store(case, gen):
    n, slots, block, heads, dim = case["rows"], case["slots"], case["block"], case["kv_heads"], case["dim"]
    codes, scales = _cache_arrays(slots, heads, dim, block, gen)
    # as many blocks as that many random rows touch, each with a row at least; the last, shorter one only if all are
    blocks = -(-slots // block)
    touched = round(blocks * (1.0 - (1.0 - n / slots) ** block))
    touched = min(max(touched, -(-n // block) + 1), n, blocks)
    full = blocks if touched == blocks or slots % block == 0 else blocks - 1
    touched = torch.randperm(full, generator=gen, device="cuda")[:touched].sort()[0]
    back = (touched[:, None] * block + torch.arange(block, device="cuda"))
    order = torch.rand(back.shape, generator=gen, device="cuda")
    order[back >= slots] = -1.0
    order.scatter_(1, order.argmax(1, keepdim=True), 2.0)
    at = back.flatten()[torch.topk(order.flatten(), n)[1]].sort()[0].int()
    back = back[back < slots].int()
    k, v = (_rows(n, heads, dim, case["dtype"], gen) for _ in range(2))
    s = dict(codes=codes, scales=scales, at=at, k=k, v=v, back=back, weight=torch.ones(slots, dtype=torch.int64, device="cuda"),
             node=torch.arange(slots, device="cuda"))
    s["k_back"], s["v_back"] = (torch.zeros(back.numel(), heads, dim, dtype=torch.float32, device="cuda") for _ in range(2))
    return s


def _prepare_admit(case, gen):
    slots, nodes, batch = case["slots"], case["nodes"], case["batch"]
    perm = torch.randperm(nodes, generator=gen, device="cuda")
    node = perm[:slots].clone()
    weight = (torch.exp(1.5 * torch.randn(slots, generator=gen, device="cuda", dtype=torch.float64)) * 2.0 ** 30).long() + 1
    weight[torch.rand(slots, generator=gen, device="cuda") < 0.1] = 1  # admitted by the last batch and not attended to
    free = torch.rand(slots, generator=gen, device="cuda") < 0.02
    node[free], weight[free] = -1, 0
    remap = torch.full((nodes,), -1, dtype=torch.int32, device="cuda")
    held = torch.nonzero(node >= 0)[:, 0]
    remap[node[held]] = held.int()
    hits = min(int(batch * case["cached"]), held.numel())
    hit = node[held[torch.randperm(held.numel(), generator=gen, device="cuda")[:hits]]]
    ids = torch.cat([hit, perm[slots:slots + batch - hits]])
    ids = ids[torch.randperm(ids.numel(), generator=gen, device="cuda")].contiguous()
    if case["repeats"]:
        ids[-case["repeats"]:] = ids[:case["repeats"]].clone()
    s = dict(remap=remap, node=node, weight=weight, ids=ids, codes=torch.zeros(slots, 2, 1, 16, dtype=torch.uint8, device="cuda"),
             scales=torch.zeros(-(-slots // 16), 1, 2, device="cuda"), remap_now=remap.clone(),
             count=torch.zeros(4, dtype=torch.int64, device="cuda"))
    for name in ("slot_of", "fresh", "fresh_slot"):
        s[name] = torch.zeros(ids.numel(), dtype=torch.int32, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------


def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": _attend_own, "store": _store_own, "admit": _admit_own}[op](s)
    return {"attend": _attend_plain, "store": _store_plain, "admit": _admit_plain}[op](s)


def _attend_own(s):
    c, dci = s["case"], s["dci"]
    n_dev = None if s["n_dev"] is None else s["n_dev"].data_ptr()
    if not c["slots"]:
        dci.dci_attn_forward(s["ctx"], s["q"], s["k"], s["v"], s["indptr"], s["src"], s["out"], s["scale"], lse=s["lse"], bias=s["bias"],
                             n_dev=n_dev, max_list=c["longest"])
        return dict(out=s["out"], lse=s["lse"])
    if c["accumulate"]:
        s["cache"].weight.copy_(s["weight"])
    dci.dci_attn_cached(s["ctx"], s["q"], s["cache"], s["indptr"], s["src"], s["out"], s["scale"], slots=s["slot_of"], lse=s["lse"],
                        bias=s["bias"], accumulate=c["accumulate"], n_dev=n_dev, max_list=c["longest"])
    got = dict(out=s["out"], lse=s["lse"])
    if c["accumulate"]:
        got["weight"] = s["cache"].weight.float() * UNIT
    return got


def _store_own(s):
    dci = s["dci"]
    dci.dci_kv_write(s["ctx"], s["cache"], s["at"], s["k"], s["v"])
    dci.dci_kv_read(s["ctx"], s["cache"], s["back"], s["k_back"], s["v_back"])
    return dict(k=s["k_back"], v=s["v_back"])


def _admit_own(s):
    dci, cache = s["dci"], s["cache"]
    s["remap_now"].copy_(s["remap"])
    cache.node.copy_(s["node"])
    cache.weight.copy_(s["weight"])
    dci.dci_kv_admit(s["ctx"], cache, s["remap_now"], s["ids"], s["slot_of"], s["fresh"], s["fresh_slot"], s["count"])
    return dict(slots=s["slot_of"], fresh=s["fresh"], fresh_slot=s["fresh_slot"], count=s["count"], remap=s["remap_now"], node=cache.node,
                weight=cache.weight)


# ---- the plain form --------------------------------------------------------------------------------


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, within the limits."""
    m, x = torch.frexp(amax)  # amax = m * 2^x, m in [0.5, 1)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX).float()


def _cached_rows(s, slot, part):
    """fp32 rows [entries, heads, dim] of the cache; part 0: keys, 1: values."""
    c = s["case"]
    x = s["codes"][slot, part, :, :c["dim"]].view(torch.float8_e4m3fn).float()
    return x * s["scales"][torch.div(slot, c["block"], rounding_mode="floor"), :, part][:, :, None]


def _attend_plain(s):
    c = s["case"]
    n, heads, kv, dim = c["rows"], c["heads"], c["kv_heads"], c["dim"]
    group = heads // kv
    out, lse = torch.zeros(c["bound"], heads, dim, device="cuda"), torch.zeros(c["bound"], heads, device="cuda")
    peak = torch.full((n, heads), -math.inf, device="cuda")
    indptr = s["indptr"][:n + 1]
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), indptr[1:] - indptr[:-1], output_size=s["src"].numel())
    src = s["src"].long()
    slot = s["slot_of"].long()[src] if c["slots"] else src
    keep = slot >= 0
    slot = slot.clamp(min=0)
    q = s["q"].float()
    z = torch.empty(src.numel(), heads, device="cuda")
    step = max(1, (1 << 29) // (heads * dim))
    for lo in range(0, src.numel(), step):
        sl, r = slot[lo:lo + step], row[lo:lo + step]
        k = _cached_rows(s, sl, 0) if c["slots"] else s["k"][sl].float()
        z[lo:lo + step] = (q[r].view(-1, kv, group, dim) * k[:, :, None, :]).sum(-1).flatten(1) * s["scale"]
    if s["bias"] is not None:
        z = z + s["bias"]
    z = torch.where(keep[:, None], z, torch.full_like(z, -math.inf))
    peak.scatter_reduce_(0, row[:, None].expand(-1, heads), z, "amax")
    peak = torch.where(torch.isinf(peak), torch.zeros_like(peak), peak)
    p = torch.exp(z - peak[row])
    total = torch.zeros(n, heads, device="cuda").index_add_(0, row, p)
    p = p / torch.where(total > 0, total, torch.ones_like(total))[row]
    for lo in range(0, src.numel(), step):
        sl, r = slot[lo:lo + step], row[lo:lo + step]
        v = _cached_rows(s, sl, 1) if c["slots"] else s["v"][sl].float()
        out.index_add_(0, r, (p[lo:lo + step].view(-1, kv, group, 1) * v[:, :, None, :]).flatten(1, 2))
    lse[:n] = torch.log(total) + peak
    got = dict(out=out.to(TYPES[c["dtype"]]), lse=lse)
    if c["accumulate"]:
        weight = s["weight"].double() * UNIT
        weight.index_add_(0, slot, torch.where(keep, p.double().sum(1), torch.zeros(1, device="cuda", dtype=torch.float64)))
        got["weight"] = weight.float()
    return got


def _store_plain(s):
    c = s["case"]
    slots, block, dim, at = c["slots"], c["block"], c["dim"], s["at"].long()
    scales = s["scales"].mT
    blocks = scales.shape[0]
    x = torch.stack([s["k"], s["v"]], 1).float()  # [n, 2, heads, dim]
    of = torch.div(at, block, rounding_mode="floor")
    amax = torch.zeros(scales.shape, device="cuda")
    amax.scatter_reduce_(0, of[:, None, None].expand(-1, 2, c["kv_heads"]), x.abs().amax(-1), "amax")
    count = torch.zeros(blocks, device="cuda").index_add_(0, of, torch.ones(at.numel(), device="cuda"))
    rows = torch.full((blocks,), float(block), device="cuda")
    rows[-1] = slots - (blocks - 1) * block
    need, old = _exponent(amax), torch.log2(scales)
    new = torch.where((count == rows)[:, None, None], need, torch.maximum(old, need))
    new = torch.where((count > 0)[:, None, None], new, old).round()
    back = s["back"].long()
    b = torch.div(back, block, rounding_mode="floor")
    held = s["codes"][back, :, :, :dim].view(torch.float8_e4m3fn).float() * torch.exp2(old[b] - new[b])[..., None]
    held = _held(held).view(torch.float8_e4m3fn).float()
    place = torch.full((slots,), -1, dtype=torch.int64, device="cuda")
    place[back] = torch.arange(back.numel(), device="cuda")
    held[place[at]] = _held(x * torch.exp2(-new[of])[..., None]).view(torch.float8_e4m3fn).float()
    y = held * torch.exp2(new[b])[..., None]
    return dict(k=y[:, 0].contiguous(), v=y[:, 1].contiguous())


def _admit_plain(s):
    remap, node, weight, ids = s["remap"].clone(), s["node"].clone(), s["weight"].clone(), s["ids"]
    n, slots = ids.numel(), node.numel()
    at = remap[ids].long()
    hit = torch.zeros(slots, dtype=torch.bool, device="cuda")
    hit[at[at >= 0]] = True
    first = torch.full((remap.numel(),), n, dtype=torch.int64, device="cuda")
    place = torch.arange(n, device="cuda")
    first.scatter_reduce_(0, ids, place, "amin")
    missed = torch.nonzero((at < 0) & (first[ids] == place))[:, 0]
    key = torch.where(hit, torch.full_like(weight, 2 ** 63 - 1), weight)
    m = min(missed.numel(), int((~hit).sum()))
    taken = torch.sort(key, stable=True)[1][:m].sort()[0]
    gone = node[taken]
    remap[gone[gone >= 0]] = -1
    placed = missed[:m]
    node[taken], weight[taken] = ids[placed], 1
    remap[ids[placed]] = taken.int()
    fresh, fresh_slot = (torch.full((n,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    fresh[:m], fresh_slot[:m] = placed.int(), taken.int()
    count = torch.stack([torch.tensor(m, device="cuda"), torch.tensor(missed.numel(), device="cuda"), hit.sum(), (gone >= 0).sum()])
    return dict(slots=remap[ids], fresh=fresh, fresh_slot=fresh_slot, count=count, remap=remap, node=node, weight=weight)


# ---- what a pass cannot do without -----------------------------------------------------------------


def _distinct(sources, entries):
    """Expected number of sources that `entries` draws of a squared uniform number name."""
    x = (np.arange(4000) + 0.5) / 4000
    return sources * float(np.mean(1.0 - np.exp(-entries / sources / (2.0 * np.sqrt(x)))))


def work(case):
    size = 4 if case.get("dtype") == "fp32" else 2
    if case["op"] == "attend":
        n, e = case["rows"], case["rows"] * case["mean"]
        rows = _distinct(case["sources"], e)
        row = 2 * case["kv_heads"] * case["dim"] * (1 if case["slots"] else size)
        moved = 2 * n * case["heads"] * case["dim"] * size + 4 * n * case["heads"] + 8 * n + 4 * e * (1 + case["bias"]) + rows * row
        if case["slots"]:
            moved += 4 * rows + 8 * case["kv_heads"] * min(rows, case["slots"] / case["block"])
        if case["accumulate"]:
            moved += 16 * rows
        return {"bytes": float(moved), "flops": 4.0 * e * case["heads"] * case["dim"]}
    if case["op"] == "store":
        width = 2 * case["kv_heads"] * case["dim"]
        blocks = -(-case["slots"] // case["block"])
        share = case["rows"] / case["slots"]
        back = case["slots"] * (1.0 - (1.0 - share) ** case["block"])
        return {"bytes": float(case["rows"] * (width * (size + 1) + 4) + back * (5 * width + 4) + 8 * case["kv_heads"] * blocks), "flops": 0.0}
    return {"bytes": float(8 * case["slots"] + case["batch"] * (8 + 4 + 4) + 28 * case["batch"] * (1 - case["cached"])), "flops": 0.0}


# ---- the definition, in 64 bits ----------------------------------------------------------------------


def _e4m3_values():
    """What the 256 codes of a sign, four exponent and three mantissa bits stand for (the largest pattern is no number)."""
    code = np.arange(256)
    exponent, mantissa = (code >> 3) & 15, code & 7
    value = np.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * 2.0 ** (exponent.astype(float) - 10))
    value = np.where((code & 127) == 127, np.nan, value)
    return torch.from_numpy(np.where(code >> 7, -value, value)).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _attend_exact, "store": _store_exact, "admit": _admit_exact}[case["op"]](s)


def _attend_exact(s):
    c = s["case"]
    n, heads, kv, dim = c["rows"], c["heads"], c["kv_heads"], c["dim"]
    bounds = s["indptr"][:n + 1].tolist()
    if n > 2_000 and max(b - a for a, b in zip(bounds, bounds[1:])) > 100:
        return None
    table = _e4m3_values()
    out = torch.zeros(c["bound"], heads, dim, dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["bound"], heads, dtype=torch.float64, device="cuda")
    weight = s["weight"].double() / 2.0 ** 32 if c["accumulate"] else None

    def keys_and_values(slot):
        if not c["slots"]:
            return s["k"][slot].double(), s["v"][slot].double()
        both = table[s["codes"][slot][..., :dim].long()] * s["scales"].mT[slot // c["block"]].double()[..., None]
        return both[..., 0, :, :], both[..., 1, :, :]

    longest = max([1] + [b - a for a, b in zip(bounds, bounds[1:])])
    at_once = max(1, min(4096, (1 << 27) // (longest * heads * dim)))
    for lo in range(0, n, at_once):  # rows side by side, lists padded to the longest
        hi = min(n, lo + at_once)
        start, length = s["indptr"][lo:hi], s["indptr"][lo + 1:hi + 1] - s["indptr"][lo:hi]
        width = max(1, int(length.max()))
        step = torch.arange(width, device="cuda")
        inside = step < length[:, None]
        entry = torch.where(inside, start[:, None] + step, torch.zeros_like(start)[:, None])
        if s["src"].numel() == 0:
            lse[lo:hi] = -math.inf
            continue
        slot = s["src"][entry].long()
        if c["slots"]:
            slot = s["slot_of"][slot].long()
        inside &= slot >= 0
        slot = slot.clamp(min=0)
        k, v = keys_and_values(slot)  # [rows, width, kv, dim]
        z = torch.empty(hi - lo, width, heads, dtype=torch.float64, device="cuda")
        for h in range(heads):
            z[:, :, h] = (s["q"][lo:hi, None, h].double() * k[:, :, h * kv // heads]).sum(-1) * s["scale"]
        if s["bias"] is not None:
            z += s["bias"][entry].double()
        z[~inside] = -math.inf
        lse[lo:hi] = torch.logsumexp(z, 1)
        p = torch.where(torch.isinf(z), torch.zeros_like(z), torch.exp(z - lse[lo:hi, None]))
        for h in range(heads):
            out[lo:hi, h] = (p[:, :, h, None] * v[:, :, h * kv // heads]).sum(1)
        if weight is not None:
            weight.index_add_(0, slot.flatten(), (p.sum(-1) * inside).flatten())
    got = dict(out=out, lse=lse)
    if weight is not None:
        got["weight"] = weight
    return got


def _store_exact(s):
    c = s["case"]
    dim, block = c["dim"], c["block"]
    table = _e4m3_values()
    held = table[s["codes"][..., :dim].long()]  # [slots, 2, heads, dim], without the scales
    at, slots = s["at"].long(), c["slots"]
    padded = -(-slots // block) * block
    new = torch.full((padded, 2, c["kv_heads"], dim), math.nan, dtype=torch.float64, device="cuda")
    new[at, 0], new[at, 1] = s["k"].double(), s["v"].double()
    written = torch.zeros(padded, dtype=torch.bool, device="cuda")
    written[at] = True
    kept = ~written
    kept[slots:] = False
    amax = torch.where(written[:, None, None], new.abs().amax(-1), torch.zeros(1, dtype=torch.float64, device="cuda"))
    amax = amax.view(-1, block, 2, c["kv_heads"]).amax(1)
    need = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -140) / 448.0)).clamp(E_MIN, E_MAX)
    need = torch.where(448.0 * torch.exp2(need - 1) >= amax, (need - 1).clamp(min=E_MIN), need)
    old = torch.log2(s["scales"].mT.double())
    e = torch.where(kept.view(-1, block).any(1)[:, None, None], torch.maximum(old, need), need)
    e = torch.repeat_interleave(e, block, 0)
    old = torch.repeat_interleave(old, block, 0)
    x = torch.where(written[:, None, None, None], new, torch.zeros(1, dtype=torch.float64, device="cuda"))
    x[:slots] = torch.where(written[:slots, None, None, None], x[:slots], held * torch.exp2(old[:slots])[..., None])
    y = x * torch.exp2(-e)[..., None]
    magnitude = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -60))).clamp(min=-6.0)
    step = torch.exp2(magnitude - 3)
    y = (torch.round(y / step) * step).clamp(-448.0, 448.0) * torch.exp2(e)[..., None]
    back = s["back"].long()
    return dict(k=y[back, 0], v=y[back, 1])


def _admit_exact(s):
    remap, node, weight, ids = (s[k].cpu().numpy().copy() for k in ("remap", "node", "weight", "ids"))
    at = remap[ids]
    protected = np.zeros(node.size, dtype=bool)
    protected[at[at >= 0]] = True
    _, first = np.unique(ids, return_index=True)
    first.sort()
    missed = first[at[first] < 0]
    open_slots = np.nonzero(~protected)[0]
    order = np.lexsort((open_slots, weight[open_slots]))
    m = min(missed.size, open_slots.size)
    taken = np.sort(open_slots[order[:m]])
    gone = node[taken]
    remap[gone[gone >= 0]] = -1
    node[taken], weight[taken] = ids[missed[:m]], 1
    remap[ids[missed[:m]]] = taken
    fresh, fresh_slot = np.full(ids.size, -1, dtype=np.int32), np.full(ids.size, -1, dtype=np.int32)
    fresh[:m], fresh_slot[:m] = missed[:m], taken
    count = np.array([m, missed.size, protected.sum(), (gone >= 0).sum()], dtype=np.int64)
    back = lambda a: torch.from_numpy(a).cuda()
    return dict(slots=back(remap[ids].astype(np.int32)), fresh=back(fresh), fresh_slot=back(fresh_slot), count=back(count), remap=back(remap),
                node=back(node), weight=back(weight))
