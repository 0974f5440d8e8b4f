"""dci_attn_forward and dci_attn_cached against the definition in 64 bits: types, head layouts, list lengths, masks, strides, splits.

Tolerances are those of attention_reference.attend: what 32-bit products, sums and exponentials can be off, and half a step of the output's
type."""
import math

import numpy as np
import pytest
import torch

from tests import attention_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def lists(lengths, sources, rng, outside=0.0):
    indptr = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    src = rng.integers(0, sources, int(indptr[-1])).astype(np.int32)
    if outside and src.size:
        src[rng.random(src.size) < outside] = rng.choice([-1, sources, sources + 5, 2 ** 31 - 1, -2 ** 31])
    return indptr, src


def rounded(a, dtype):
    return torch.from_numpy(a).to(TYPES[dtype])


def check(out, lse, want, n, dtype):
    got = out[:n].float().cpu().numpy().astype(np.float64)
    tol = want[3] + ref.HALF_STEP[dtype] * np.abs(want[0]) + ref.SMALLEST[dtype]
    bad = ~(np.abs(got - want[0]) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[0][bad][:4], tol[bad][:4])
    if lse is not None:
        got = lse[:n].cpu().numpy().astype(np.float64)
        empty = np.isneginf(want[1])
        assert np.array_equal(np.isneginf(got), empty)
        assert (np.abs(got[~empty] - want[1][~empty]) <= want[4][~empty]).all()


def make_cache(dci, n_slots, heads, dim, block, rng):
    """A cache of random codes (no NaN) and scales, and its values in float64 [n_slots, 2, heads, dim]."""
    width, blocks = -(-dim // 16) * 16, -(-n_slots // block)
    codes = rng.integers(0, 256, (n_slots, 2, heads, width)).astype(np.uint8)
    codes[(codes & 127) == 127] = 0x38
    codes[..., dim:] = 0
    scales = 2.0 ** rng.integers(-9, -5, (blocks, heads, 2)).astype(np.float64)
    values = ref.e4m3_values()[codes[..., :dim]] * np.repeat(scales, block, 0)[:n_slots].transpose(0, 2, 1)[..., None]
    weight = rng.integers(1, 2 ** 40, n_slots).astype(np.int64)
    dev = lambda a: torch.from_numpy(a).cuda()
    return dci.KvCache.from_arrays(dev(codes), dev(scales.astype(np.float32)), dev(weight), dev(np.arange(n_slots, dtype=np.int64)), dim, block), values


def cached_case(dci, ctx, lengths, heads, kv, dim, dtype, seed, block=16, n_slots=300, bias_heads=0, by_slot=False, max_list=0, accumulate=True):
    rng = np.random.default_rng(seed)
    n, sources = len(lengths), 200
    indptr, src = lists(lengths, n_slots if by_slot else sources, rng, outside=0.05)
    cache, values = make_cache(dci, n_slots, kv, dim, block, rng)
    slots = rng.permutation(n_slots)[:sources].astype(np.int32)
    slots[rng.random(sources) < 0.1] = -1
    slots[7] = n_slots  # outside
    where = src.astype(np.int64)
    if by_slot:
        where = np.where((where >= 0) & (where < n_slots), where, -1)
    else:
        inside = (where >= 0) & (where < sources)
        where = np.where(inside, slots[np.where(inside, where, 0)], -1)
        where = np.where((where >= 0) & (where < n_slots), where, -1)
    if max_list:
        where = where.copy()
        for i in range(n):
            where[indptr[i] + max_list:indptr[i + 1]] = -1
    q = rounded(rng.standard_normal((n, heads, dim)).astype(np.float32), dtype)
    bias = None
    if bias_heads:
        bias = rng.standard_normal((src.size, bias_heads)).astype(np.float32)
        bias[rng.random(bias.shape) < 0.15] = -np.inf
    scale = 1.0 / math.sqrt(dim)
    want = ref.attend(q.double().numpy(), values[:, 0], values[:, 1], indptr, where, np.float64(np.float32(scale)),
                      None if bias is None else bias.astype(np.float64))
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    out = torch.full((n, heads, dim), float("nan"), dtype=TYPES[dtype], device="cuda")
    lse = torch.full((n, heads), float("nan"), device="cuda")
    before = cache.weight.cpu().numpy().copy()
    dci.dci_attn_cached(ctx, q.cuda(), cache, dev(indptr), dev(src), out, scale, slots=None if by_slot else dev(slots), lse=lse,
                        bias=dev(bias), accumulate=accumulate, max_list=max_list)
    ctx.sync()
    check(out, lse, want, n, dtype)
    added = (cache.weight.cpu().numpy() - before).astype(np.float64) / 2.0 ** 32
    if not accumulate:
        assert (added == 0).all()
        return
    keep = where >= 0
    expect, tol = np.zeros(n_slots), np.zeros(n_slots)
    np.add.at(expect, where[keep], want[2][keep].sum(1))
    # an entry's sum over the heads in fp32 (one rounding per head), and rounded to the unit in at most `heads` parts
    np.add.at(tol, where[keep], want[5][keep].sum(1) + want[2][keep].sum(1) * (heads + 1) * ref.U + heads * 2.0 ** -33)
    assert (np.abs(added - expect) <= tol).all()


LENGTHS = [0, 1, 2, 3, 15, 16, 17, 0, 63, 64, 5, 31, 0]


@pytest.mark.parametrize("heads,kv,dim,dtype", [
    (1, 1, 1, "fp32"), (1, 1, 16, "bf16"), (4, 4, 64, "fp32"), (4, 4, 64, "bf16"), (4, 4, 64, "fp16"), (3, 3, 41, "fp16"), (8, 2, 32, "bf16"),
    (6, 1, 80, "fp32"), (5, 5, 7, "bf16"), (2, 1, 128, "fp16"), (16, 2, 200, "bf16"), (1, 1, 256, "fp32"), (20, 20, 64, "bf16"), (9, 3, 17, "fp32"),
    (128, 128, 16, "fp16"), (24, 8, 128, "bf16")])
def test_cached_lists_of_a_sampled_block(heads, kv, dim, dtype):
    import paper_2503_01281_amd as dci
    cached_case(dci, dci.Context(0), LENGTHS, heads, kv, dim, dtype, seed=heads * 1000 + dim, max_list=64)


@pytest.mark.parametrize("block", [1, 2, 32, 64])
@pytest.mark.parametrize("bias_heads", [0, 1, 4])
@pytest.mark.parametrize("by_slot", [False, True])
def test_cached_scales_biases_and_slots(block, bias_heads, by_slot):
    import paper_2503_01281_amd as dci
    cached_case(dci, dci.Context(0), LENGTHS, 4, 2, 48, "fp32", seed=block + bias_heads, block=block, n_slots=257, bias_heads=bias_heads, by_slot=by_slot)


# lists that are cut: begin and end at every place relative to the multiples of 64, empty and short ones between them
CUT = [64, 65, 0, 128, 1, 700, 0, 0, 66, 63, 129, 5, 320, 64, 191, 0, 257]


@pytest.mark.parametrize("heads,kv,dim,dtype,bias_heads", [
    (4, 4, 64, "bf16", 0), (1, 1, 16, "fp32", 1), (8, 2, 128, "fp16", 8), (3, 3, 41, "fp32", 3), (32, 8, 128, "bf16", 0), (12, 2, 256, "fp32", 1),
    (20, 20, 64, "bf16", 20)])
def test_cached_long_lists_are_cut_and_joined(heads, kv, dim, dtype, bias_heads):
    import paper_2503_01281_amd as dci
    cached_case(dci, dci.Context(0), CUT, heads, kv, dim, dtype, seed=dim, bias_heads=bias_heads)


# query heads that share key heads, where long lists go through the matrix instructions: three to eight heads at a time, 64, 128 and 256 columns
@pytest.mark.parametrize("heads,kv,dim,dtype", [
    (4, 1, 64, "bf16"), (4, 1, 64, "fp16"), (4, 1, 64, "fp32"), (3, 1, 128, "fp32"), (10, 2, 128, "fp16"), (12, 2, 128, "bf16"), (21, 3, 64, "fp32"),
    (8, 1, 256, "bf16"), (16, 2, 256, "fp32"), (9, 1, 64, "bf16"), (16, 1, 128, "fp16"), (40, 2, 64, "bf16")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_cached_long_lists_of_shared_key_heads(heads, kv, dim, dtype, accumulate):
    import paper_2503_01281_amd as dci
    cached_case(dci, dci.Context(0), CUT, heads, kv, dim, dtype, seed=heads, accumulate=accumulate)
    cached_case(dci, dci.Context(0), [0, 95, 96, 97, 31, 1, 500], heads, kv, dim, dtype, seed=dim, block=1, by_slot=True, accumulate=accumulate)


@pytest.mark.parametrize("lengths", [[1], [0], [64], [65], [0, 0, 3000, 0], [1000] * 3, [70] * 40])
@pytest.mark.parametrize("accumulate", [False, True])
def test_cached_few_rows(lengths, accumulate):
    import paper_2503_01281_amd as dci
    cached_case(dci, dci.Context(0), lengths, 4, 4, 64, "fp32", seed=len(lengths), accumulate=accumulate)


@pytest.mark.parametrize("max_list", [1, 5, 16, 64, 65, 100, 128, 320, 699, 700, 10 ** 6])
@pytest.mark.parametrize("accumulate", [False, True])
def test_entries_beyond_max_list_do_not_count(max_list, accumulate):
    """Lists of up to 700 entries, of which the first max_list count."""
    import paper_2503_01281_amd as dci
    cached_case(dci, dci.Context(0), CUT, 4, 4, 32, "bf16", seed=3, max_list=max_list, accumulate=accumulate)


@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 4, 64, "fp32"), (4, 4, 64, "bf16"), (8, 2, 128, "fp16"), (3, 3, 41, "fp16"), (3, 1, 41, "bf16"),
                                                (2, 2, 7, "fp32"), (1, 1, 250, "fp32"), (16, 4, 256, "bf16"), (5, 5, 24, "bf16")])
@pytest.mark.parametrize("strided", [False, True])
def test_dense_rows(heads, kv, dim, dtype, strided):
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(dim + heads)
    n, sources = len(CUT), 90
    indptr, src = lists(CUT, sources, rng, outside=0.05)
    where = np.where((src >= 0) & (src < sources), src, -1).astype(np.int64)

    def rows(count, h):
        """[count, h, dim] on the GPU: in one piece, or with rows further apart and not on 16 bytes."""
        wide = torch.from_numpy(rng.standard_normal((count, h * dim + 9)).astype(np.float32)).to(TYPES[dtype]).cuda()
        if strided:
            return wide[:, 3:3 + h * dim].unflatten(1, (h, dim))
        return wide[:, :h * dim].contiguous().view(count, h, dim)

    q, k, v = rows(n, heads), rows(sources, kv), rows(sources, kv)
    want = ref.attend(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), indptr, where, np.float64(np.float32(0.3)))
    out = rows(n, heads)
    around = out.clone()
    lse = torch.full((n, heads), float("nan"), device="cuda")
    whole = out._base.clone() if strided else None
    for max_list in (0, 700):
        dci.dci_attn_forward(ctx, q, k, v, torch.from_numpy(indptr).cuda(), torch.from_numpy(src).cuda(), out, 0.3, lse=lse, max_list=max_list)
        ctx.sync()
        check(out, lse, want, n, dtype)
        out.copy_(around)
        lse.fill_(float("nan"))
    if strided:  # what lies between the rows is as it was
        now = out._base
        assert torch.equal(now[:, :3], whole[:, :3]) and torch.equal(now[:, 3 + heads * dim:], whole[:, 3 + heads * dim:])


def test_rows_behind_the_count_are_left_alone():
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(5)
    lengths = [3, 0, 70, 9, 200, 4]
    indptr, src = lists(lengths, 50, rng)
    q, k, v = (torch.from_numpy(rng.standard_normal((m, 4, 64)).astype(np.float32)).cuda() for m in (6, 50, 50))
    want = ref.attend(*(t.double().cpu().numpy() for t in (q, k, v)), indptr, src.astype(np.int64), 0.125)
    indptr_dev = torch.from_numpy(indptr).cuda()
    for n in (0, 1, 3, 5, 6, 9):
        rows = min(n, 6)
        ptr = indptr_dev.clone()
        ptr[rows + 1:] = -77  # behind the last row anything may stand
        out, lse = torch.full((6, 4, 64), 5.0, device="cuda"), torch.full((6, 4), 6.0, device="cuda")
        n_dev = torch.tensor([n], dtype=torch.int64, device="cuda")
        dci.dci_attn_forward(ctx, q, k, v, ptr, torch.from_numpy(src).cuda(), out, 0.125, lse=lse, n_dev=n_dev.data_ptr())
        ctx.sync()
        assert (out[rows:] == 5.0).all() and (lse[rows:] == 6.0).all()
        if rows:
            check(out, lse, [w[:rows] for w in want[:2]] + [None] + [w[:rows] for w in want[3:5]], rows, "fp32")


@pytest.mark.parametrize("rows,edges,sources", [(3, 0, 5), (3, 0, 0), (3, 9, 0), (3, 700, 0), (0, 0, 5), (0, 0, 0)])
@pytest.mark.parametrize("bias_heads", [0, 1, 4])
def test_calls_with_nothing_to_attend_to(rows, edges, sources, bias_heads):
    """No rows, no entries, no sources: tensors without elements, whose addresses are null, are taken as what they are."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    heads, dim = 4, 64
    cache, _ = make_cache(dci, 50, heads, dim, 16, np.random.default_rng(1))
    before = cache.weight.clone()
    indptr = torch.linspace(0, edges, rows + 1).long().cuda() if rows else torch.zeros(1, dtype=torch.int64, device="cuda")
    src = (torch.arange(edges, dtype=torch.int32) % 50).cuda()
    bias = torch.zeros(edges, bias_heads, device="cuda") if bias_heads else None
    q = torch.randn(rows, heads, dim, device="cuda")
    kv = torch.randn(sources, heads, dim, device="cuda")
    slots = torch.arange(sources, dtype=torch.int32, device="cuda")
    for cached in (False, True):
        for max_list in (0, 64):
            out, lse = torch.full_like(q, 7.0), torch.full((rows, heads), 7.0, device="cuda")
            if cached:
                dci.dci_attn_cached(ctx, q, cache, indptr, src, out, 0.125, slots=slots, lse=lse, bias=bias, accumulate=True, max_list=max_list)
            else:
                dci.dci_attn_forward(ctx, q, kv, kv, indptr, src, out, 0.125, lse=lse, bias=bias, max_list=max_list)
            ctx.sync()
            assert (out == 0).all() and torch.isneginf(lse).all() and torch.equal(cache.weight, before)


@pytest.mark.parametrize("length", [10, 500])
@pytest.mark.parametrize("cached", [False, True])
def test_left_out_entries_may_hold_anything(length, cached):
    """Rows that only left-out entries name hold NaN and infinities; the result is that without the entries, bit for bit."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(6)
    n, sources, heads, dim = 4, 64, 2, 32
    indptr, src = lists([length] * n, sources, rng)
    q = torch.from_numpy(rng.standard_normal((n, heads, dim)).astype(np.float32)).cuda()
    k, v = (rng.standard_normal((sources, heads, dim)).astype(np.float32) for _ in range(2))
    bias = rng.standard_normal((src.size, heads)).astype(np.float32)
    bias[src >= 48, :] = -np.inf
    bias[(src >= 40) & (src < 48), 1] = -np.inf  # left out for one head, not for the other
    k[40:48, 1], v[40:48, 1] = np.nan, np.inf
    clean_k, clean_v = k.copy(), v.copy()
    k[48:], v[48:] = np.nan, np.nan
    k[50], v[50] = np.inf, -np.inf
    clean_k[40:48, 1], clean_v[40:48, 1] = 1.0, 1.0
    clean_k[48:], clean_v[48:] = 0.0, 0.0
    dev = lambda a: torch.from_numpy(a).cuda()
    got = []
    for kk, vv in ((k, v), (clean_k, clean_v)):
        out, lse = torch.empty(n, heads, dim, device="cuda"), torch.empty(n, heads, device="cuda")
        if cached:
            cache = dci.KvCache(ctx, sources, heads, dim, 1)
            dci.dci_kv_write(ctx, cache, torch.arange(sources, dtype=torch.int32, device="cuda"), dev(kk), dev(vv))
            dci.dci_attn_cached(ctx, q, cache, dev(indptr), dev(src), out, 0.2, lse=lse, bias=dev(bias), accumulate=True)
            got.append((out, lse, cache.weight))
        else:
            dci.dci_attn_forward(ctx, q, dev(kk), dev(vv), dev(indptr), dev(src), out, 0.2, lse=lse, bias=dev(bias))
            got.append((out, lse))
        ctx.sync()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.isfinite(got[0][0]).all()


@pytest.mark.parametrize("length", [5, 300])
def test_masks_of_the_lowest_number_and_numbers_that_are_none(length):
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(7)
    lowest = float(np.finfo(np.float32).min)
    indptr, src = lists([length] * 5, 30, rng)
    q, k, v = (rng.standard_normal((m, 1, 16)).astype(np.float32) for m in (5, 30, 30))
    bias = np.zeros((src.size, 1), dtype=np.float32)
    bias[:length] = lowest                 # row 0: all of them: the mean of the values
    bias[length:2 * length - 1] = lowest   # row 1: all but the last
    bias[2 * length:3 * length] = -np.inf  # row 2: nothing left
    k[int(src[3 * length])] = np.nan       # row 3 (and whoever names it) is NaN
    dev = lambda a: torch.from_numpy(a).cuda()
    out, lse = torch.empty(5, 1, 16, device="cuda"), torch.empty(5, 1, device="cuda")
    k_clean = np.nan_to_num(k)
    for kk in (k_clean, k):
        dci.dci_attn_forward(ctx, dev(q), dev(kk), dev(v), dev(indptr), dev(src), out, 0.25, lse=lse, bias=dev(bias))
        ctx.sync()
        got = out.cpu().numpy()[:, 0]
        rows = [i for i in range(5) if not (kk is k and (k[src[indptr[i]:indptr[i + 1]]] != k[src[indptr[i]:indptr[i + 1]]]).any())]
        if 0 in rows:  # a mean of `length` numbers of size 5 at most: length + 8 roundings
            assert np.abs(got[0] - v[src[:length], 0].astype(np.float64).mean(0)).max() <= (4 * length + 32) * ref.U * 5
        if 1 in rows:  # weight 1 and weights 0: exact
            assert np.array_equal(got[1], v[src[2 * length - 1], 0])
        assert (got[2] == 0).all() and float(lse[2]) == -math.inf
    assert np.isnan(got[3]).all() and math.isnan(float(lse[3]))


def test_many_entries_take_longer_chunks():
    """More entries than 4,096 wavefronts have chunks of 64 for: chunks of 128 and more; sums in 64 bits by row."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(8)
    lengths = np.array([300_000, 5, 0, 129, 128, 256, 257, 100_001, 300, 63, 200_000])
    indptr, src = lists(lengths, 5_000, rng)
    q, k, v = (rng.standard_normal((m, 1, 16)).astype(np.float32) for m in (len(lengths), 5_000, 5_000))
    dev = lambda a: torch.from_numpy(a).cuda()
    out, lse = torch.empty(len(lengths), 1, 16, device="cuda"), torch.empty(len(lengths), 1, device="cuda")
    dci.dci_attn_forward(ctx, dev(q), dev(k), dev(v), dev(indptr), dev(src), out, 0.25, lse=lse)
    ctx.sync()
    want = ref.attend(q.astype(np.float64), k.astype(np.float64), v.astype(np.float64), indptr, src.astype(np.int64), 0.25)
    check(out, lse, want, len(lengths), "fp32")


def test_many_entries_of_shared_key_heads():
    import paper_2503_01281_amd as dci
    lengths = np.array([150_000, 5, 0, 513, 512, 100_001, 511, 64, 63, 1025])
    cached_case(dci, dci.Context(0), lengths, 4, 1, 64, "bf16", seed=11, n_slots=5_000, accumulate=False)


def test_a_side_stream_and_a_graph():
    """A call on another stream than the current one waits for nothing but that stream; captured once, it replays with new inputs."""
    import paper_2503_01281_amd as dci
    side = torch.cuda.Stream()
    ctx = dci.Context(0, stream=side)
    rng = np.random.default_rng(9)
    indptr, src = lists([5, 300, 0, 64, 70], 100, rng)
    dev = lambda a: torch.from_numpy(a).cuda()
    with torch.cuda.stream(side):
        cache, values = make_cache(dci, 100, 2, 64, 16, rng)
        ptr, s = dev(indptr), dev(src)
        q, out, lse = torch.empty(5, 4, 64, device="cuda"), torch.empty(5, 4, 64, device="cuda"), torch.empty(5, 4, device="cuda")
        base = cache.weight.clone()
        q.copy_(dev(rng.standard_normal((5, 4, 64)).astype(np.float32)))

        def step():
            cache.weight.copy_(base)
            dci.dci_attn_cached(ctx, q, cache, ptr, s, out, 0.125, lse=lse, accumulate=True)

        step()  # sizes the workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for replay in range(4):
            x = rng.standard_normal((5, 4, 64)).astype(np.float32)
            q.copy_(dev(x))
            step()
            ctx.sync()
            eager = [t.clone() for t in (out, lse, cache.weight)]
            out.fill_(float("nan")), lse.fill_(float("nan")), cache.weight.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, (out, lse, cache.weight))), replay
            want = ref.attend(x.astype(np.float64), values[:, 0], values[:, 1], indptr, src.astype(np.int64), 0.125)
            check(out, lse, want, 5, "fp32")


def test_refusals():
    import paper_2503_01281_amd as dci
    from paper_2503_01281_amd import binding as b
    ctx = dci.Context(0)
    lib = ctx.lib
    t = {k: torch.zeros(64, 64, device="cuda") for k in ("q", "out", "k", "v")}
    ptr, src = torch.zeros(65, dtype=torch.int64, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    cache = dci.KvCache(ctx, 32, 2, 32)

    def args(**kw):
        a = b._Attn(4, None, ptr.data_ptr(), src.data_ptr(), 8, 16, 0, 0, 2, 2, 32, 1.0, t["q"].data_ptr(), 64, t["out"].data_ptr(), 64, None, None, 0)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    import ctypes as C

    def dense(a, k_stride=64, k=t["k"].data_ptr(), v=t["v"].data_ptr()):
        return lib.dci_attn_forward(ctx.handle, C.byref(a) if a is not None else None, k, k_stride, v, 64)

    assert dense(args()) == 0
    assert lib.dci_attn_cached(ctx.handle, C.byref(args()), C.byref(cache.c), None, 1) in (0, -2)
    for bad in (dict(n_rows=-1), dict(n_edges=-1), dict(n_src=-1), dict(max_list=-1), dict(n_heads=0), dict(kv_heads=0), dict(n_heads=3),
                dict(head_dim=0), dict(head_dim=257), dict(n_heads=130, kv_heads=130), dict(dtype=3), dict(dtype=-1), dict(indptr=None), dict(src=None),
                dict(q=None), dict(out=None), dict(q_stride=63), dict(out_stride=0), dict(q=t["q"].data_ptr() + 2), dict(out=t["out"].data_ptr() + 1),
                dict(bias_heads=1), dict(bias=t["v"].data_ptr()), dict(bias=t["v"].data_ptr(), bias_heads=3)):
        assert dense(args(**bad)) == -1, bad
        assert lib.dci_attn_cached(ctx.handle, C.byref(args(**bad)), C.byref(cache.c), None, 0) == -1, bad
    assert dense(args(n_rows=2 ** 31)) == -4 and dense(args(n_src=2 ** 31)) == -4 and dense(args(n_edges=2 ** 39)) == -4
    assert dense(None) == -1 and dense(args(), k_stride=63) == -1 and dense(args(), k=None) == -1 and dense(args(), v=t["v"].data_ptr() + 2) == -1
    assert dense(args(n_rows=0, q=None, out=None, indptr=None)) == 0
    assert lib.dci_attn_cached(ctx.handle, C.byref(args(kv_heads=1)), C.byref(cache.c), None, 0) == -1
    assert lib.dci_attn_cached(ctx.handle, C.byref(args(head_dim=16)), C.byref(cache.c), None, 0) == -1
    assert lib.dci_attn_cached(ctx.handle, C.byref(args()), None, None, 0) == -1
    no_weight = dci.KvCache.from_arrays(cache.codes, cache.scales, None, None, 32, 16)
    assert lib.dci_attn_cached(ctx.handle, C.byref(args()), C.byref(no_weight.c), None, 1) == -1
    assert lib.dci_attn_cached(ctx.handle, C.byref(args()), C.byref(no_weight.c), None, 0) == 0
    # a workspace that is too small is named with what is needed
    small = dci.Context(0)
    a = args(n_edges=64)
    assert lib.dci_attn_workspace_bytes(C.byref(a), 0) == 0 and lib.dci_attn_workspace_bytes(C.byref(a), 1) == 0
    a = args(n_edges=65)
    assert 0 < lib.dci_attn_workspace_bytes(C.byref(a), 0) < lib.dci_attn_workspace_bytes(C.byref(a), 1)
    assert lib.dci_attn_cached(small.handle, C.byref(a), C.byref(cache.c), None, 1) == -2
    assert small.last_required()[2] == lib.dci_attn_workspace_bytes(C.byref(a), 1)
    ctx.sync()


def test_a_graph_keeps_the_workspace_it_was_captured_with():
    """A later call that needs more workspace takes a new one; the graph's own stays, and is nobody else's."""
    import paper_2503_01281_amd as dci
    side = torch.cuda.Stream()
    ctx = dci.Context(0, stream=side)
    rng = np.random.default_rng(10)

    def inputs(lengths):
        indptr, src = lists(lengths, 50, rng)
        return [torch.from_numpy(a).cuda() for a in (indptr, src)] + [torch.randn(len(lengths), 2, 32, device="cuda"), torch.empty(len(lengths), 2, 32, device="cuda")]

    with torch.cuda.stream(side):
        k, v = torch.randn(50, 2, 32, device="cuda"), torch.randn(50, 2, 32, device="cuda")
        small, large = inputs([100, 200, 3]), inputs([2000] * 20)

        def call(x):
            dci.dci_attn_forward(ctx, x[2], k, v, x[0], x[1], x[3], 0.2)

        call(small)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(small)
        held = ctx._ws
        for replay in range(3):
            call(large)
            assert ctx._ws is not held
            mine = [torch.full((1 << 18,), 3.0, device="cuda") for _ in range(64)]  # what would lie where the old workspace did
            call(small)
            ctx.sync()
            want = small[3].clone()
            small[3].fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            ctx.sync()
            assert torch.equal(small[3], want) and all(bool((m == 3.0).all()) for m in mine), replay
