"""Attention over lists, the 8-bit key/value cache and its admission, plainly and in 64 bits (numpy), with the error that 32-bit sums may
have beside each output.  No code of the library."""
import math

import numpy as np

U = 2.0 ** -24  # half a unit in the last place of an fp32 number, relative
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}  # rounding to the type, relative
SMALLEST = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}  # the types' smallest steps


def e4m3_values():
    code = np.arange(256)
    exponent, mantissa = (code >> 3) & 15, code & 7
    value = np.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * 2.0 ** (exponent.astype(float) - 10))
    value[(code & 127) == 127] = np.nan
    return np.where(code >> 7, -value, value)


def to_e4m3(x):
    """The nearest e4m3 numbers (ties to the even mantissa), at most 448, NaN for what is no number; as float64."""
    x = np.asarray(x, dtype=np.float64)
    good = np.isfinite(x)
    y = np.where(good, x, 0.0)
    _, e = np.frexp(np.where(y == 0, 1.0, np.abs(y)))  # |y| = f * 2^e, f in [0.5, 1)
    step = 2.0 ** (np.maximum(e - 1, -6) - 3)
    y = np.clip(np.rint(y / step) * step, -448.0, 448.0)
    return np.where(good, y, np.nan)


def need_exponent(amax):
    if amax == 0:
        return -100
    e = math.ceil(math.log2(amax / 448.0)) - 2
    while 448.0 * 2.0 ** e < amax:
        e += 1
    return min(max(e, -100), 119)


def attend(q, k, v, indptr, rows_of_entry, scale, bias=None):
    """q [n, heads, dim], k, v [rows, kv_heads, dim] in float64; rows_of_entry [n_edges]: the row of k and v that an entry names, -1: left out;
    bias [n_edges, 1 or heads].  Returns out, lse, p [n_edges, heads] and the errors out, lse and p may have when every product, sum
    and exponential is one of fp32."""
    n, heads, dim = q.shape
    group = heads // (k.shape[1] if k.size else heads)
    out, lse = np.zeros_like(q), np.full((n, heads), -np.inf)
    out_err, lse_err = np.zeros_like(q), np.zeros((n, heads))
    p_all, p_err = np.zeros((len(rows_of_entry), heads)), np.zeros((len(rows_of_entry), heads))
    for i in range(n):
        e = np.arange(indptr[i], indptr[i + 1])
        for h in range(heads):
            keep = rows_of_entry[e] >= 0
            b = None
            if bias is not None:
                b = bias[e, h if bias.shape[1] > 1 else 0]
                keep = keep & ~np.isneginf(b)
            if not keep.any():
                continue
            r = rows_of_entry[e][keep]
            kk, vv = k[r, h // group], v[r, h // group]
            z = kk @ q[i, h] * scale
            # a dot product of dim terms, the scale, the key's scale and the bias: dim + 4 roundings of at most the sum of the magnitudes
            dz = (dim + 4) * U * (np.abs(kk) @ np.abs(q[i, h]) * abs(scale))
            if b is not None:
                z = z + b[keep]
                dz = dz + U * np.abs(z)
            m = z.max()
            p = np.exp(z - m)
            total = p.sum()
            lse[i, h] = m + math.log(total)
            p /= total
            # each weight: its score's error and the joint one of the others; the difference to the maximum and its product with log2 e
            # rounded (3 roundings of at most 1.5 times the difference), an exponential of two units; up to a rescaling and an addition for
            # each of the entries before it, in numerator and sum; a division
            worst = float((p * dz).sum())
            rel = dz + worst + U * (5 * np.abs(z - m) + 5 * float((p * np.abs(z - m)).sum()) + 4 * len(r) + 24)
            p_all[e[keep], h] = p
            p_err[e[keep], h] = p * rel
            out[i, h] = p @ vv
            out_err[i, h] = (p * rel) @ np.abs(vv) + U * 2 * np.abs(out[i, h])
            lse_err[i, h] = worst + U * (5 * float((p * np.abs(z - m)).sum()) + 4 * len(r) + 24 + 2 * abs(lse[i, h]) + 2 * abs(m))
    return out, lse, p_all, out_err, lse_err, p_err


def write(held, exponents, slots, k, v, n_slots, block):
    """held [n_slots, 2, heads, dim]: e4m3 numbers before the scales; exponents [blocks, 2, heads], None-like -1000 where there is none yet.
    Both are changed as a write of rows k, v [n, heads, dim] to `slots` changes them."""
    rows = np.stack([k, v], 1).astype(np.float64)
    by_block = {}
    for i, s in enumerate(slots):
        if 0 <= s < n_slots:
            by_block.setdefault(int(s) // block, []).append((i, int(s)))
    for b, entries in by_block.items():
        of_block = range(b * block, min((b + 1) * block, n_slots))
        kept = [s for s in of_block if s not in {s for _, s in entries}]
        for kind in range(2):
            for h in range(held.shape[2]):
                x = rows[[i for i, _ in entries], kind, h]
                finite = np.abs(x[np.isfinite(x)])
                need, old = need_exponent(float(finite.max()) if finite.size else 0.0), int(exponents[b, kind, h])
                e = max(need, old) if kept and old != -1000 else need
                if kept and old != -1000 and e > old:
                    held[kept, kind, h] = to_e4m3(held[kept, kind, h] * 2.0 ** (old - e))
                for i, s in entries:
                    held[s, kind, h] = to_e4m3(rows[i, kind, h] * 2.0 ** -e)
                exponents[b, kind, h] = e


def admit(remap, node, weight, ids):
    """Changes remap, node and weight as an admission of the batch `ids` does; returns slots, fresh, fresh_slots, counts."""
    n, n_slots = len(ids), len(node)
    hit, first = set(), {}
    for i, v in enumerate(ids):
        if not 0 <= v < len(remap):
            continue
        if remap[v] >= 0:
            hit.add(int(remap[v]))
        else:
            first.setdefault(int(v), i)
    missed = sorted(first.values())
    order = sorted((int(weight[s]), s) for s in range(n_slots) if s not in hit)
    m = min(len(missed), len(order))
    taken = sorted(s for _, s in order[:m])
    evicted = 0
    for j, s in enumerate(taken):
        if node[s] >= 0:
            remap[node[s]] = -1
            evicted += 1
        node[s], weight[s] = ids[missed[j]], 1
        remap[ids[missed[j]]] = s
    slots = np.array([remap[v] if 0 <= v < len(remap) else -1 for v in ids], dtype=np.int32)
    fresh, fresh_slots = np.full(n, -1, dtype=np.int32), np.full(n, -1, dtype=np.int32)
    fresh[:m], fresh_slots[:m] = missed[:m], taken
    return slots, fresh, fresh_slots, np.array([m, len(missed), len(hit), evicted], dtype=np.int64)
