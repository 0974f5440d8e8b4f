"""The 8-bit key/value cache against its definition: writing, reading, admission by eviction, and a model's step over all of them.  Codes,
scales, read rows and everything that admission writes are defined to the bit."""
import math

import numpy as np
import pytest
import torch

from tests import attention_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def held_by(cache):
    """(e4m3 numbers [n_slots, 2, heads, dim] before the scales, exponents [blocks, 2, heads])"""
    scales = cache.scales.cpu().numpy().astype(np.float64).transpose(0, 2, 1)
    exponents = np.where(scales == 0, -1000, np.log2(np.where(scales == 0, 1.0, scales)))
    return ref.e4m3_values()[cache.codes.cpu().numpy()[..., :cache.head_dim]], exponents


def some_rows(rng, n, heads, dim, dtype, spread=3.0):
    """Rows of differing magnitudes, now and then all zeros or with numbers that are none."""
    x = rng.standard_normal((n, heads, dim)) * 2.0 ** np.rint(rng.standard_normal((n, 1, 1)) * spread)
    x[rng.random((n, heads)) < 0.1] = 0.0
    x[rng.random(x.shape) < 0.003] = np.nan
    x[rng.random(x.shape) < 0.003] = np.inf
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])


def compare(cache, held, exponents):
    got, got_e = held_by(cache)
    assert np.array_equal(got_e, exponents)
    assert np.array_equal(np.nan_to_num(got, nan=1e9), np.nan_to_num(held, nan=1e9))
    assert (cache.codes.cpu().numpy()[..., cache.head_dim:] == 0).all()


@pytest.mark.parametrize("heads,dim,dtype", [(4, 64, "bf16"), (4, 64, "fp32"), (1, 1, "fp32"), (3, 41, "fp16"), (2, 128, "bf16"), (1, 256, "fp32"),
                                             (8, 16, "fp16"), (5, 24, "bf16"), (2, 200, "fp32")])
@pytest.mark.parametrize("block", [1, 4, 16, 64])
def test_writes_and_reads(heads, dim, dtype, block):
    """A fill, then writes of single rows, of half the rows and of whole blocks; strided and unaligned rows."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(block * 1000 + dim)
    n_slots = 203
    cache = dci.KvCache(ctx, n_slots, heads, dim, block)
    held, exponents = held_by(cache)
    assert (exponents == -1000).all() and (held == 0).all()
    for turn, slots in enumerate([np.arange(n_slots), np.array([0]), np.array([n_slots - 1]), np.sort(rng.permutation(n_slots)[:100]),
                                  np.arange(64, 128), np.sort(rng.permutation(n_slots)[:9]), np.arange(150, n_slots), np.arange(0, n_slots, 3)]):
        n = len(slots)
        k, v = some_rows(rng, n, heads, dim, dtype), some_rows(rng, n, heads, dim, dtype)
        if turn % 2:  # rows apart, on addresses that are not multiples of 16 bytes
            hold = [torch.full((n, heads * dim + 5), 7.0, dtype=k.dtype, device="cuda") for _ in range(2)]
            kd, vd = (t[:, 1:1 + heads * dim].unflatten(1, (heads, dim)) for t in hold)
            kd.copy_(k), vd.copy_(v)
        else:
            kd, vd = k.cuda(), v.cuda()
        at = np.concatenate([slots, [-1, n_slots, -5][:turn % 4]]).astype(np.int32)  # entries outside, behind all others
        if len(at) > n:
            pad = torch.zeros(len(at) - n, heads, dim, dtype=k.dtype, device="cuda")
            kd, vd = torch.cat([kd, pad]), torch.cat([vd, pad])
        dci.dci_kv_write(ctx, cache, dev(at), kd, vd)
        ctx.sync()
        ref.write(held, exponents, slots, k.double().numpy(), v.double().numpy(), n_slots, block)
        compare(cache, held, exponents)
    values = held * 2.0 ** np.repeat(exponents, block, 0)[:n_slots][..., None]
    order = rng.integers(-3, n_slots + 3, 300).astype(np.int32)
    inside = (order >= 0) & (order < n_slots)
    for out_type in TYPES:
        for strided in (False, True):
            hold = [torch.full((300, heads * dim + 3), 7.0, dtype=TYPES[out_type], device="cuda") for _ in range(2)]
            k, v = (t[:, 1:1 + heads * dim].unflatten(1, (heads, dim)) if strided else t[:, :heads * dim].contiguous().view(300, heads, dim) for t in hold)
            dci.dci_kv_read(ctx, cache, dev(order), k, v)
            ctx.sync()
            for kind, t in enumerate((k, v)):
                want = torch.from_numpy(values[order[inside], kind]).to(TYPES[out_type])  # one rounding of numbers that fp32 holds exactly
                got = t.cpu()[inside]
                assert torch.equal(torch.nan_to_num(got, 1e4), torch.nan_to_num(want, 1e4))
                assert (t.cpu()[~inside] == 7.0).all()


def test_scales_at_the_ends_of_the_number_range():
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    big, tiny = float(np.finfo(np.float32).max), float(2.0 ** -149)
    rows = np.zeros((12, 1, 16), dtype=np.float32)
    rows[0, 0, 0], rows[1, 0, 0], rows[2, 0, 0] = big, tiny, 448.0
    rows[3, 0, 0], rows[4, 0, 0], rows[5, 0, 0] = np.nextafter(np.float32(448.0), np.float32(500)), 2.0 ** -126, -big
    rows[6, 0, :3] = [np.nan, np.inf, -np.inf]
    rows[7, 0, :2] = [1.75 * 2.0 ** 127, -1.75 * 2.0 ** 127]
    rows[8, 0, 0], rows[9, 0, 0], rows[10, 0, :2] = 448.0 * 2.0 ** -100, 448.0 * 2.0 ** -101, [2.0 ** -130, -3.0e-39]
    for block in (1, 2):
        cache = dci.KvCache(ctx, 12, 1, 16, block)
        held, exponents = held_by(cache)
        dci.dci_kv_write(ctx, cache, dev(np.arange(12, dtype=np.int32)), dev(rows), dev(-rows))
        ctx.sync()
        ref.write(held, exponents, np.arange(12), rows, -rows, 12, block)
        compare(cache, held, exponents)
        k, v = torch.empty(12, 1, 16, device="cuda"), torch.empty(12, 1, 16, device="cuda")
        dci.dci_kv_read(ctx, cache, dev(np.arange(12, dtype=np.int32)), k, v)
        ctx.sync()
        want = held[:, 0] * 2.0 ** np.repeat(exponents[:, 0], block, 0)[..., None]
        assert np.array_equal(np.nan_to_num(k.cpu().numpy().astype(np.float64), nan=1e9), np.nan_to_num(want, nan=1e9))


def test_every_16_bit_number_is_rounded_as_defined():
    """All bf16 and fp16 numbers that are some, a number to a slot with blocks of one slot, and 64 to a block."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    for dtype in ("bf16", "fp16"):
        x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(TYPES[dtype]).view(-1, 1, 16)
        for block in (1, 64):
            n = x.shape[0]
            cache = dci.KvCache(ctx, n, 1, 16, block)
            held, exponents = held_by(cache)
            dci.dci_kv_write(ctx, cache, torch.arange(n, dtype=torch.int32, device="cuda"), x.cuda(), x.flip(0).contiguous().cuda())
            ctx.sync()
            ref.write(held, exponents, np.arange(n), x.double().numpy(), x.flip(0).double().numpy(), n, block)
            compare(cache, held, exponents)


def test_counts_on_the_gpu_and_slots_that_do_not_ascend():
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    cache = dci.KvCache(ctx, 64, 2, 32, 16)
    rng = np.random.default_rng(1)
    rows = rng.standard_normal((10, 2, 32)).astype(np.float32)
    slots = np.array([1, 2, 3, 20, 21, 40, 50, 51, 62, 63], dtype=np.int32)
    held, exponents = held_by(cache)
    n_dev = torch.tensor([4], dtype=torch.int64, device="cuda")
    dci.dci_kv_write(ctx, cache, dev(slots), dev(rows), dev(rows), n_dev=n_dev.data_ptr())
    ctx.sync()
    ref.write(held, exponents, slots[:4], rows[:4], rows[:4], 64, 16)
    compare(cache, held, exponents)
    k, v = torch.full((10, 2, 32), 9.0, device="cuda"), torch.full((10, 2, 32), 9.0, device="cuda")
    dci.dci_kv_read(ctx, cache, dev(slots), k, v, n_dev=n_dev.data_ptr())
    ctx.sync()
    assert (k[4:] == 9.0).all() and (v[4:] == 9.0).all() and (k[:4] != 9.0).all()
    for bad in ([5, 5], [6, 5], [3, -1, 4], [40, 2]):
        dci.dci_kv_write(ctx, cache, dev(np.array(bad, dtype=np.int32)), dev(rows[:len(bad)]), dev(rows[:len(bad)]))
        with pytest.raises(dci.DciError) as err:
            ctx.sync()
        assert err.value.code == -1 and "ascending" in str(err.value)
        ctx.sync()  # reported once


def admission_state(rng, n_nodes, n_slots, free, weights):
    node = rng.permutation(n_nodes)[:n_slots].astype(np.int64)
    weight = weights(n_slots).astype(np.int64) + 1
    empty = rng.random(n_slots) < free
    node[empty], weight[empty] = -1, 0
    remap = np.full(n_nodes, -1, dtype=np.int32)
    remap[node[~empty]] = np.nonzero(~empty)[0]
    return remap, node, weight


def run_admit(dci, ctx, remap, node, weight, ids, n_dev=None):
    n = len(ids)
    cache = dci.KvCache.from_arrays(torch.zeros(len(node), 2, 1, 16, dtype=torch.uint8, device="cuda"), torch.zeros(len(node), 1, 2, device="cuda"),
                                    dev(weight), dev(node), 16, 1)
    r, out = dev(remap), [torch.full((n,), -9, dtype=torch.int32, device="cuda") for _ in range(3)]
    counts = torch.full((4,), -9, dtype=torch.int64, device="cuda")
    count = None if n_dev is None else torch.tensor([n_dev], dtype=torch.int64, device="cuda")
    dci.dci_kv_admit(ctx, cache, r, dev(ids), *out, counts, n_dev=None if count is None else count.data_ptr())
    ctx.sync()
    return [t.cpu().numpy() for t in out + [counts, r, cache.node, cache.weight]]


def check_admit(dci, ctx, remap, node, weight, ids, n_dev=None):
    got = run_admit(dci, ctx, remap, node, weight, ids, n_dev)
    n = len(ids) if n_dev is None else min(n_dev, len(ids))
    remap, node, weight = remap.copy(), node.copy(), weight.copy()
    slots, fresh, fresh_slots, counts = ref.admit(remap, node, weight, ids[:n])
    assert np.array_equal(got[3], counts), (got[3], counts)
    assert np.array_equal(got[0][:n], slots) and (got[0][n:] == -9).all()
    for g, w in ((got[1], fresh), (got[2], fresh_slots)):
        assert np.array_equal(g[:n], w) and (g[n:] == -1).all()
    for g, w in zip(got[4:], (remap, node, weight)):
        assert np.array_equal(g, w)


WEIGHTS = {
    "alike": lambda rng: lambda n: np.zeros(n),
    "small": lambda rng: lambda n: rng.integers(0, 200, n),
    "of all sizes": lambda rng: lambda n: np.exp2(rng.uniform(0, 62.9, n)),
    "close together": lambda rng: lambda n: 2 ** 40 + rng.integers(0, 5, n),
    "equal and large": lambda rng: lambda n: np.full(n, 2 ** 62 + 12345),
    "as of sums": lambda rng: lambda n: np.exp(rng.standard_normal(n)) * 2 ** 32,
    "two bits apart": lambda rng: lambda n: 2 ** 50 + 2 ** rng.integers(0, 40, n),
}


@pytest.mark.parametrize("weights", WEIGHTS)
@pytest.mark.parametrize("n_slots,batch", [(1, 1), (1, 5), (31, 40), (700, 300), (5000, 2500), (5000, 1), (9001, 12000)])
def test_admission(weights, n_slots, batch):
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(n_slots + batch)
    n_nodes = 15_000
    for free in (0.0, 0.1, 1.0):
        remap, node, weight = admission_state(rng, n_nodes, n_slots, free, WEIGHTS[weights](rng))
        held = node[node >= 0]
        hits = held[rng.permutation(len(held))[:batch // 3]]
        ids = np.concatenate([hits, rng.integers(0, n_nodes, batch - len(hits))]).astype(np.int64)  # repeats among them
        rng.shuffle(ids)
        if batch > 3:
            ids[rng.integers(0, batch, 2)] = [-1, n_nodes]  # ids of no node
        check_admit(dci, ctx, remap, node, weight, ids)


def test_admission_without_a_choice():
    """Nothing to do, all hits, all slots hit, one node over and over, a batch counted on the GPU."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(2)
    remap, node, weight = admission_state(rng, 1000, 300, 0.0, WEIGHTS["as of sums"](rng))
    check_admit(dci, ctx, remap, node, weight, np.zeros(0, dtype=np.int64))
    check_admit(dci, ctx, remap, node, weight, node.copy())
    check_admit(dci, ctx, remap, node, weight, np.concatenate([node, np.arange(1000)]))
    outside = np.nonzero(remap < 0)[0].astype(np.int64)
    check_admit(dci, ctx, remap, node, weight, np.full(2000, outside[0]))
    check_admit(dci, ctx, remap, node, weight, np.concatenate([node[:299], outside]))
    for n in (0, 1, 77, 300, 5000):
        check_admit(dci, ctx, remap, node, weight, rng.permutation(1000)[:300].astype(np.int64), n_dev=n)


def test_admission_again_and_again_keeps_the_books():
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(3)
    remap, node, weight = np.full(4000, -1, dtype=np.int32), np.full(900, -1, dtype=np.int64), np.zeros(900, dtype=np.int64)
    for turn in range(8):
        ids = np.unique((4000 * rng.random(600) ** 3).astype(np.int64))
        rng.shuffle(ids)
        got = run_admit(dci, ctx, remap, node, weight, ids)
        ref.admit(remap, node, weight, ids)
        for g, w in zip(got[4:], (remap, node, weight)):
            assert np.array_equal(g, w)
        held = np.nonzero(node >= 0)[0]
        assert np.array_equal(remap[node[held]], held) and (remap >= 0).sum() == len(held)
        weight[remap[ids]] += rng.integers(0, 2 ** 34, len(ids))


def test_large_caches_and_batches():
    """More tiles than one workgroup scans at once; the reference is vectorised."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(4)
    n_nodes, n_slots, batch = 2_000_000, 1_200_007, 500_003
    remap, node, weight = admission_state(rng, n_nodes, n_slots, 0.01, WEIGHTS["as of sums"](rng))
    ids = rng.permutation(n_nodes)[:batch].astype(np.int64)
    got = run_admit(dci, ctx, remap, node, weight, ids)
    at = remap[ids]
    hit = np.zeros(n_slots, dtype=bool)
    hit[at[at >= 0]] = True
    missed = np.nonzero(at < 0)[0]
    open_slots = np.nonzero(~hit)[0]
    m = min(len(missed), len(open_slots))
    taken = np.sort(open_slots[np.lexsort((open_slots, weight[open_slots]))[:m]])
    gone = node[taken]
    remap[gone[gone >= 0]] = -1
    node[taken], weight[taken] = ids[missed[:m]], 1
    remap[ids[missed[:m]]] = taken
    assert got[3].tolist() == [m, len(missed), int(hit.sum()), int((gone >= 0).sum())]
    assert np.array_equal(got[0], remap[ids])
    assert np.array_equal(got[1][:m], missed[:m]) and np.array_equal(got[2][:m], taken) and (got[1][m:] == -1).all() and (got[2][m:] == -1).all()
    for g, w in zip(got[4:], (remap, node, weight)):
        assert np.array_equal(g, w)


@pytest.mark.parametrize("dim,dtype", [(64, "fp32"), (64, "bf16"), (41, "fp16"), (41, "fp32")])
def test_a_read_of_more_than_the_last_level_cache(dim, dtype):
    """One large read gives, to the bit, what reads of a few rows give; entries outside the cache leave their rows alone."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    heads, n_slots, bytes_ = 4, 1000, 4 if dtype == "fp32" else 2
    n = (300 << 20) // (2 * heads * dim * bytes_)
    rng = np.random.default_rng(dim)
    cache = dci.KvCache(ctx, n_slots, heads, dim, 16)
    dci.dci_kv_write(ctx, cache, dev(np.arange(n_slots, dtype=np.int32)), some_rows(rng, n_slots, heads, dim, dtype).cuda(),
                     some_rows(rng, n_slots, heads, dim, dtype).cuda())
    one = [torch.empty(n_slots, heads, dim, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    dci.dci_kv_read(ctx, cache, dev(np.arange(n_slots, dtype=np.int32)), *one)
    at = torch.from_numpy(rng.integers(-5, n_slots + 5, n).astype(np.int32)).cuda()
    got = [torch.full((n, heads * dim + 1), 7.0, dtype=TYPES[dtype], device="cuda")[:, :heads * dim].unflatten(1, (heads, dim)) for _ in range(2)]
    dci.dci_kv_read(ctx, cache, at, *got)
    ctx.sync()
    inside = (at >= 0) & (at < n_slots)
    whole = torch.int32 if bytes_ == 4 else torch.int16
    for g, o in zip(got, one):
        want = torch.where(inside[:, None, None], o[at.long().clamp(0, n_slots - 1)], torch.full((), 7.0, dtype=o.dtype, device="cuda"))
        assert torch.equal(g.contiguous().view(whole), want.view(whole))


def test_a_cache_beyond_4_gib():
    """Codes behind the 32-bit range of offsets: written, read and attended to."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    n_slots = 9_000_000  # of 512 bytes
    cache = dci.KvCache(ctx, n_slots, 4, 64, 16)
    rng = np.random.default_rng(5)
    slots = np.array([0, 5, 4_194_303, 4_194_304, 8_388_607, 8_388_608, 8_999_990, 8_999_999], dtype=np.int32)
    rows = [rng.standard_normal((8, 4, 64)).astype(np.float32) for _ in range(2)]
    dci.dci_kv_write(ctx, cache, dev(slots), dev(rows[0]), dev(rows[1]))
    k, v = torch.empty(8, 4, 64, device="cuda"), torch.empty(8, 4, 64, device="cuda")
    dci.dci_kv_read(ctx, cache, dev(slots), k, v)
    q = rng.standard_normal((1, 4, 64)).astype(np.float32)
    out = torch.empty(1, 4, 64, device="cuda")
    dci.dci_attn_cached(ctx, dev(q), cache, dev(np.array([0, 8])), dev(slots), out, 0.125, accumulate=True)
    ctx.sync()
    # the first block of a fill: every group of slots that share a block has a scale of its own
    for kind, t in enumerate((k, v)):
        for b in np.unique(slots // 16):
            of = slots // 16 == b
            x = rows[kind][of].astype(np.float64)
            e = np.array([ref.need_exponent(float(np.abs(x[:, h]).max())) for h in range(4)])
            assert np.array_equal(t.cpu().numpy()[of], ref.to_e4m3(x * 2.0 ** -e[None, :, None]) * 2.0 ** e[None, :, None])
    want = ref.attend(q.astype(np.float64), k.double().cpu().numpy(), v.double().cpu().numpy(), [0, 8], np.arange(8), 0.125)
    assert (np.abs(out.cpu().numpy() - want[0]) <= want[3] + ref.U * np.abs(want[0])).all()
    weights = cache.weight[torch.from_numpy(slots).long().cuda()].cpu().numpy() / 2.0 ** 32
    assert (np.abs(weights - want[2].sum(1)) <= want[5].sum(1) + want[2].sum(1) * 5 * ref.U + 2.0 ** -31).all()
    assert int((cache.weight != 0).sum()) == 8


def test_batches_of_a_model_follow_their_cache(tiny):
    """What they are for, together: batches are sampled; their input nodes get slots, by eviction once the cache is full; the rows of the new
    ones are gathered, projected and written; the last hop's rows attend over the cache, which adds up the weights that decide the next eviction.
    Every step is checked against the definition, the later layer's dense attention too."""
    import paper_2503_01281_amd as dci
    from tests import gpu_util as gu
    w = tiny["w"]
    ctx = dci.Context(0)
    g = gu.make_graph(tiny["indptr"], tiny["indices"], tiny["feat"])
    heads, dim, n_slots, block = 4, 16, 4096, 16
    width = heads * dim
    rng = np.random.default_rng(6)
    wq, wk, wv = (dev((rng.standard_normal((w.feat_dim, width)) / 8).astype(np.float32)) for _ in range(3))
    cache = dci.KvCache(ctx, n_slots, heads, dim, block)
    held, exponents = held_by(cache)
    remap_now = torch.full((w.num_nodes,), -1, dtype=torch.int32, device="cuda")
    remap, node, weight = np.full(w.num_nodes, -1, dtype=np.int32), np.full(n_slots, -1, dtype=np.int64), np.zeros(n_slots, dtype=np.int64)
    blk = dci.Blocks(ctx, w.num_nodes, w.batch_size, w.fanouts)
    cap = blk.cap_nodes[-1]
    slots, fresh, fresh_slots = (torch.empty(cap, dtype=torch.int32, device="cuda") for _ in range(3))
    counts = torch.zeros(4, dtype=torch.int64, device="cuda")
    x = torch.zeros(cap, w.feat_dim, device="cuda")
    hop = w.n_hops - 1
    rows = blk.cap_nodes[hop]
    out, lse = torch.zeros(rows, heads, dim, device="cuda"), torch.zeros(rows, heads, device="cuda")
    evictions = 0
    for batch in range(5):
        seeds = gu.dev(tiny["seeds"][batch * w.batch_size:(batch + 1) * w.batch_size])
        dci.dci_sample_khop(ctx, g, None, seeds, batch, w.fanouts, w.rng_seed, blk)
        dci.dci_kv_admit(ctx, cache, remap_now, blk.nodes, slots, fresh, fresh_slots, counts, n_dev=blk.n_input_dev())
        dci.dci_gather_features(ctx, g, None, blk.nodes, cap, x, n_dev=blk.n_input_dev())
        ctx.sync()
        m = int(counts[0])
        new = x[fresh[:m].long()]
        k, v = (new @ wk).view(m, heads, dim), (new @ wv).view(m, heads, dim)
        dci.dci_kv_write(ctx, cache, fresh_slots[:m], k, v)
        n = blk.n_nodes()
        q = (x[:rows] @ wq).view(rows, heads, dim)
        before = cache.weight.cpu().numpy()
        dci.dci_attn_cached(ctx, q, cache, blk.blk_indptr[hop], blk.blk_src[hop], out, 0.25, slots=slots, lse=lse, accumulate=True,
                            n_dev=blk.counts.data_ptr() + 8 * hop, max_list=w.fanouts[hop])
        got = gu.blocks_to_host(ctx, blk)
        # admission
        s_want, f_want, fs_want, c_want = ref.admit(remap, node, weight, got["nodes"])
        assert np.array_equal(counts.cpu().numpy(), c_want) and np.array_equal(slots.cpu().numpy()[:n[-1]], s_want)
        assert np.array_equal(fresh.cpu().numpy()[:n[-1]], f_want) and np.array_equal(fresh_slots.cpu().numpy()[:n[-1]], fs_want)
        assert np.array_equal(before, weight) and np.array_equal(cache.node.cpu().numpy(), node) and np.array_equal(remap_now.cpu().numpy(), remap)
        evictions += int(c_want[3])
        # the written rows
        ref.write(held, exponents, fs_want[:m], k.double().cpu().numpy(), v.double().cpu().numpy(), n_slots, block)
        compare(cache, held, exponents)
        # attention
        values = held * np.where(exponents == -1000, 0.0, 2.0 ** exponents).repeat(block, 0)[:n_slots][..., None]
        where = s_want[got["blk_src"][hop]].astype(np.int64)
        want = ref.attend(q[:n[hop]].double().cpu().numpy(), values[:, 0], values[:, 1], got["blk_indptr"][hop], where, 0.25)
        assert (np.abs(out[:n[hop]].cpu().numpy() - want[0]) <= want[3] + ref.U * np.abs(want[0])).all()
        after = cache.weight.cpu().numpy()
        expect, tol = np.zeros(n_slots), np.zeros(n_slots)
        np.add.at(expect, where[where >= 0], want[2][where >= 0].sum(1))
        np.add.at(tol, where[where >= 0], want[5][where >= 0].sum(1) + want[2][where >= 0].sum(1) * 5 * ref.U + 2.0 ** -31)
        assert (np.abs((after - before) / 2.0 ** 32 - expect) <= tol).all()
        weight[:] = after
        # the layer behind it attends to the rows of the batch
        hidden = out[:n[hop]].contiguous()
        q1, out1 = hidden[:n[hop - 1]].contiguous(), torch.empty(n[hop - 1], heads, dim, device="cuda")
        dci.dci_attn_forward(ctx, q1, hidden, hidden, blk.blk_indptr[hop - 1][:n[hop - 1] + 1].contiguous(), blk.blk_src[hop - 1], out1, 0.25,
                             max_list=w.fanouts[hop - 1])
        ctx.sync()
        h64 = hidden.double().cpu().numpy()
        want = ref.attend(h64[:n[hop - 1]], h64, h64, got["blk_indptr"][hop - 1], got["blk_src"][hop - 1].astype(np.int64), 0.25)
        assert (np.abs(out1.cpu().numpy() - want[0]) <= want[3] + ref.U * np.abs(want[0])).all()
    assert evictions > 0


def test_a_step_replays_from_a_graph():
    """Admission, the new rows' write, attention: captured once, replayed over changing batches, against the eager calls."""
    import paper_2503_01281_amd as dci
    side = torch.cuda.Stream()
    ctx = dci.Context(0, stream=side)
    rng = np.random.default_rng(7)
    n_nodes, n_slots, batch, heads, dim = 3000, 512, 300, 2, 32
    with torch.cuda.stream(side):
        table = dev(rng.standard_normal((2, n_nodes, heads, dim)).astype(np.float32))
        cache = dci.KvCache(ctx, n_slots, heads, dim, 16)
        remap = torch.full((n_nodes,), -1, dtype=torch.int32, device="cuda")
        ids = torch.zeros(batch, dtype=torch.int64, device="cuda")
        slots, fresh, fresh_slots = (torch.zeros(batch, dtype=torch.int32, device="cuda") for _ in range(3))
        counts = torch.zeros(4, dtype=torch.int64, device="cuda")
        indptr = dev(np.arange(0, batch + 1, 10))
        src = dev(np.arange(batch, dtype=np.int32))
        q, out = dev(rng.standard_normal((30, heads, dim)).astype(np.float32)), torch.empty(30, heads, dim, device="cuda")
        state = [cache.codes, cache.scales, cache.weight, cache.node, remap]

        def step():
            dci.dci_kv_admit(ctx, cache, remap, ids, slots, fresh, fresh_slots, counts)
            rows = table[:, ids[fresh.clamp(min=0).long()]]
            dci.dci_kv_write(ctx, cache, fresh_slots, rows[0], rows[1])
            dci.dci_attn_cached(ctx, q, cache, indptr, src, out, 0.2, slots=slots, accumulate=True, max_list=10)

        keep = [t.clone() for t in state]
        step()
        for t, s in zip(state, keep):
            t.copy_(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for replay in range(6):
            ids.copy_(dev(rng.permutation(n_nodes)[:batch].astype(np.int64)))
            keep = [t.clone() for t in state]
            step()
            ctx.sync()
            eager = [t.clone() for t in state + [slots, fresh, fresh_slots, counts, out]]
            for t, s in zip(state, keep):
                t.copy_(s)
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            ctx.sync()
            for a, b in zip(eager, state + [slots, fresh, fresh_slots, counts, out]):
                assert torch.equal(a, b), replay
        assert int(counts[3]) > 0


def test_refusals():
    import ctypes as C

    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    lib = ctx.lib
    cache = dci.KvCache(ctx, 32, 2, 32)
    rows = torch.zeros(8, 64, device="cuda")
    slots = torch.arange(8, dtype=torch.int32, device="cuda")
    p, s = rows.data_ptr(), slots.data_ptr()
    for call in (lib.dci_kv_write, lib.dci_kv_read):
        assert call(ctx.handle, C.byref(cache.c), s, 8, None, 0, p, 64, p, 64) == 0
        assert call(ctx.handle, C.byref(cache.c), None, 0, None, 0, None, 64, None, 64) == 0
        for bad in ((s, -1, None, 0, p, 64, p, 64), (None, 8, None, 0, p, 64, p, 64), (s, 8, None, 3, p, 64, p, 64), (s, 8, None, 0, None, 64, p, 64),
                    (s, 8, None, 0, p, 63, p, 64), (s, 8, None, 0, p, 64, p, 0), (s, 8, None, 0, p + 2, 64, p, 64), (s, 8, None, 1, p, 64, p + 1, 64)):
            assert call(ctx.handle, C.byref(cache.c), *bad) == -1, bad
        assert call(ctx.handle, C.byref(cache.c), s, 2 ** 31, None, 0, p, 64, p, 64) == -4
        assert call(ctx.handle, None, s, 8, None, 0, p, 64, p, 64) == -1

    def changed(**kw):
        c = type(cache.c).from_buffer_copy(cache.c)
        for k, v in kw.items():
            setattr(c, k, v)
        return C.byref(c)

    for bad in (dict(n_slots=0), dict(n_slots=2 ** 31), dict(block=0), dict(block=3), dict(block=128), dict(kv_heads=0), dict(kv_heads=129),
                dict(head_dim=0), dict(head_dim=257), dict(codes=None), dict(scales=None), dict(codes=cache.codes.data_ptr() + 8),
                dict(scales=cache.scales.data_ptr() + 4)):
        assert lib.dci_kv_clear(ctx.handle, changed(**bad)) == -1, bad
        assert lib.dci_kv_write(ctx.handle, changed(**bad), s, 8, None, 0, p, 64, p, 64) == -1, bad
    nodes, remap, counts = (torch.zeros(64, dtype=t, device="cuda") for t in (torch.int64, torch.int32, torch.int64))
    ctx.ensure_workspace(lib.dci_kv_admit_workspace_bytes(32, 64))
    n, r, c = nodes.data_ptr(), remap.fill_(-1).data_ptr(), counts.data_ptr()
    good = (r, 64, n, 8, None, s, s, s, c)
    for at, value in ((0, None), (1, 0), (2, None), (3, -1), (5, None), (6, None), (7, None), (8, None)):
        bad = list(good)
        bad[at] = value
        assert lib.dci_kv_admit(ctx.handle, C.byref(cache.c), *bad) == -1, (at, value)
    assert lib.dci_kv_admit(ctx.handle, changed(weight=None), *good) == -1
    assert lib.dci_kv_admit(ctx.handle, changed(node=None), *good) == -1
    assert lib.dci_kv_admit(ctx.handle, C.byref(cache.c), r, 2 ** 31, n, 8, None, s, s, s, c) == -4
    small = dci.Context(0)
    assert lib.dci_kv_admit(small.handle, C.byref(cache.c), *good) == -2
    assert small.last_required()[2] == lib.dci_kv_admit_workspace_bytes(32, 8)
    ctx.sync()
