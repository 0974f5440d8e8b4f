"""Attention over lists where its arithmetic and its launches end: infinite keys at every way that a head's columns lie on lanes, no
sources, more pieces than one launch has workgroups for, workspaces sized for another call, weights of few bits.

Tolerances are those of attention_reference.attend, or derived where they are used."""
import math

import numpy as np
import pytest
import torch

from tests import attention_reference as ref
from tests.test_gpu_attention import TYPES, check, lists, rounded

pytestmark = pytest.mark.gpu


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


# widths that fill their lanes (8, 64, 256), leave lanes without columns (24, 40, 80, 96) or end inside a piece (9, 41, 97, 200)
@pytest.mark.parametrize("dim", [8, 9, 24, 40, 41, 64, 80, 96, 97, 200, 256])
@pytest.mark.parametrize("heads,kv,dtype,bias_heads", [(3, 3, "fp32", 0), (4, 2, "fp32", 4), (8, 2, "fp32", 0), (2, 2, "bf16", 1), (4, 2, "fp16", 0),
                                                       (4, 1, "fp16", 4)])
def test_infinite_keys_of_dense_rows(dim, heads, kv, dtype, bias_heads):
    """A key whose score is -inf has weight 0, wherever in the row its infinity stands; one whose score is none makes the row none."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(dim * 100 + heads)
    sources, lengths = 120, [5, 0, 64, 17, 130, 1, 300, 40]
    indptr, src = lists(lengths, sources, rng)
    src[indptr[:-1][np.array(lengths) > 0]] = 0  # every list begins with a source whose key is finite
    n = len(lengths)
    q, k, v = (rounded(rng.standard_normal((m, h, dim)).astype(np.float32), dtype) for m, h in ((n, heads), (sources, kv), (sources, kv)))
    q = q.abs() + 0.25  # positive: a key of -inf gives a score of -inf
    gone = np.zeros(sources, dtype=bool)
    for s in range(1, sources):
        if rng.random() < 0.4:
            gone[s] = True
            k[s, :, rng.integers(max(0, dim - 17), dim) if s % 3 else rng.integers(dim)] = -math.inf
    bias = rng.standard_normal((src.size, bias_heads)).astype(np.float32) if bias_heads else None
    where = np.where(gone[src], -1, src).astype(np.int64)
    finite = torch.where(torch.isinf(k), torch.zeros_like(k), k)
    scale = 1.0 / math.sqrt(dim)
    want = ref.attend(q.double().numpy(), finite.double().numpy(), v.double().numpy(), indptr, where, np.float64(np.float32(scale)),
                      None if bias is None else bias.astype(np.float64))

    def call():
        out, lse = torch.full((n, heads, dim), 7.0, dtype=TYPES[dtype], device="cuda"), torch.full((n, heads), 7.0, device="cuda")
        dci.dci_attn_forward(ctx, q.cuda(), k.cuda(), v.cuda(), dev(indptr), dev(src), out, scale, lse=lse, bias=dev(bias))
        ctx.sync()
        return out, lse

    out, lse = call()
    check(out, lse, want, n, dtype)
    s = int(src[indptr[2] + 3])  # a source of row 2: infinities of both signs, no score
    if dim > 1 and s != 0:
        k[s, :, dim - 1], k[s, :, 0] = -math.inf, math.inf
        named = np.array([s in src[indptr[i]:indptr[i + 1]] for i in range(n)])
        out, lse = call()
        assert torch.isnan(out.float()).all(-1).cpu().numpy()[named].all() and torch.isnan(lse).cpu().numpy()[named].all()
        assert not torch.isnan(out.float()).any(-1).cpu().numpy()[~named].any()


@pytest.mark.parametrize("heads,kv,dim", [(4, 1, 64), (16, 2, 128), (3, 1, 256), (4, 4, 64), (8, 2, 32)])
@pytest.mark.parametrize("rows,each", [(1, 65), (3, 700), (40, 90)])
def test_long_lists_without_sources(heads, kv, dim, rows, each):
    """Slots without elements: entries, long lists of heads that share keys among them, name nothing."""
    import ctypes as C

    import paper_2503_01281_amd as dci
    from paper_2503_01281_amd import binding as b
    from tests.test_gpu_attention import make_cache
    ctx = dci.Context(0)
    cache, _ = make_cache(dci, 50, kv, dim, 16, np.random.default_rng(rows))
    before = cache.weight.clone()
    indptr = torch.arange(0, rows * each + 1, each, device="cuda")
    src = (torch.arange(rows * each, dtype=torch.int32) % 50).cuda()
    q = torch.randn(rows, heads, dim, device="cuda")
    for through in ("binding", "library"):
        out, lse = torch.full_like(q, 7.0), torch.full((rows, heads), 7.0, device="cuda")
        if through == "binding":
            dci.dci_attn_cached(ctx, q, cache, indptr, src, out, 0.125, slots=torch.empty(0, dtype=torch.int32, device="cuda"), lse=lse, accumulate=True)
        else:
            a = b._attn_args(q, kv, 0, indptr, src, out, 0.125, lse, None, None, 0)
            ctx.check(ctx.lib.dci_attn_cached(ctx.handle, C.byref(a), C.byref(cache.c), src.data_ptr(), 1))  # not null, and none of it is a slot
        ctx.sync()
        assert (out == 0).all() and torch.isneginf(lse).all() and torch.equal(cache.weight, before)


def test_more_chunks_and_heads_than_a_launch_has_workgroups():
    """67 million entries, 128 heads: with chunks of 512 the join would need 16.8 million workgroups, 2^32 lanes and more."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(12)
    n, each, heads, dim, sources = 131_300, 512, 128, 16, 100
    gen = torch.Generator(device="cuda").manual_seed(12)
    indptr = torch.arange(0, (n + 1) * each, each, device="cuda") - each // 2  # lists that begin in the middle of a chunk
    indptr[0] = 0
    src = torch.randint(sources, (int(indptr[-1]),), generator=gen, device="cuda", dtype=torch.int32)
    q = torch.randn(n, heads, dim, generator=gen, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn(sources, heads, dim, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    out, lse = torch.full_like(q, float("nan")), torch.full((n, heads), float("nan"), device="cuda")
    dci.dci_attn_forward(ctx, q, k, v, indptr, src, out, 0.25, lse=lse)
    ctx.sync()
    assert torch.isfinite(lse).all() and torch.isfinite(out).all()
    for i in np.unique(np.concatenate([[0, 1, n - 2, n - 1, 2 ** 17 - 1, 2 ** 17], rng.integers(0, n, 3)])):
        b, e = int(indptr[i]), int(indptr[i + 1])
        want = ref.attend(q[i:i + 1].double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), [0, e - b],
                          src[b:e].cpu().numpy().astype(np.int64), 0.25)
        check(out[i:i + 1], lse[i:i + 1], want, 1, "bf16")


def test_a_workspace_sized_by_the_largest_call():
    """A caller of the library who takes the workspace of the largest call has room for all smaller ones: here half as many, longer chunks need half."""
    import ctypes as C

    import paper_2503_01281_amd as dci
    from paper_2503_01281_amd import binding as b
    rng = np.random.default_rng(13)
    heads, dim, sources = 4, 64, 100
    k, v = (torch.from_numpy(rng.standard_normal((sources, heads, dim)).astype(np.float32)).cuda() for _ in range(2))
    for largest, smaller in ((16_400, 16_384), (262_208, 262_144), (300_000, 40_000), (262_208, 65)):
        ctx, args = dci.Context(0), {}
        for edges in (largest, smaller):
            indptr, src = lists([edges // 3, 0, edges - edges // 3], sources, rng)
            q, out = torch.randn(3, heads, dim, device="cuda"), torch.empty(3, heads, dim, device="cuda")
            args[edges] = (b._attn_args(q, heads, sources, dev(indptr), dev(src), out, 0.125, None, None, None, 0), q, out, indptr, src)
        held = [dev(a[4]) for a in args.values()], [dev(a[3]) for a in args.values()]
        for (a, *_), s, p in zip(args.values(), *held):
            a.src, a.indptr = s.data_ptr(), p.data_ptr()
        ctx.ensure_workspace(ctx.lib.dci_attn_workspace_bytes(C.byref(args[largest][0]), 0))
        for edges, (a, q, out, indptr, src) in args.items():
            ctx.check(ctx.lib.dci_attn_forward(ctx.handle, C.byref(a), k.data_ptr(), heads * dim, v.data_ptr(), heads * dim))
            ctx.sync()
            want = ref.attend(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), indptr, src.astype(np.int64), 0.125)
            check(out, None, want, 3, "fp32")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv", [(3, 1), (5, 1), (6, 1), (7, 1), (8, 1), (9, 1), (13, 1), (16, 2)])
def test_weights_of_shared_key_heads_keep_the_bits_of_fp32(heads, kv, dim):
    """Long lists of which two entries are left: values 0 with score 0 and values V with score -d, out = V / (1 + exp(d)), so that an error of the
    second weight is the output's.  Scores are exact (one product each).  In units of 2^-24: 2.5 each for the weight's exponential, for that of a
    rescaling and for that of a join (two in the last place, and the rounded argument times 0.1); 3 for the products with those in the accumulator,
    and as many again, 10.5, in the sum; 5 for the additions of parts, pieces and the sum; 3 for the reciprocal and its product: 32 at most.  Two bf16
    numbers can be off by 64 (2^-18)."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(heads * 10 + dim)
    n, each, n_slots = 250, 70, 4
    codes = np.zeros((n_slots, 2, kv, dim), dtype=np.uint8)
    codes[1, 0, :, 0] = 0x38  # a key of (1, 0, 0, ...)
    codes[1, 1] = rng.integers(0x30, 0x60, (kv, dim))
    scales = np.ones((n_slots, kv, 2), dtype=np.float32)
    cache = dci.KvCache.from_arrays(dev(codes), dev(scales), None, None, dim, 1)
    values = ref.e4m3_values()[codes]
    src = np.full((n, each), -1, dtype=np.int32)
    for i in range(n):
        src[i, np.sort(rng.permutation(each)[:2])] = rng.permutation(2)
    indptr = np.arange(0, n * each + 1, each)
    q = np.zeros((n, heads, dim), dtype=np.float32)
    q[:, :, 0] = -rng.uniform(0.002, 0.1, (n, heads))
    want = ref.attend(q.astype(np.float64), values[:, 0], values[:, 1], indptr, src.ravel().astype(np.int64), 1.0)
    for dtype in ("fp32", "bf16"):
        if dtype == "bf16":
            q = rounded(q, dtype).float().numpy()
            want = ref.attend(q.astype(np.float64), values[:, 0], values[:, 1], indptr, src.ravel().astype(np.int64), 1.0)
        out, lse = torch.empty(n, heads, dim, dtype=TYPES[dtype], device="cuda"), torch.empty(n, heads, device="cuda")
        dci.dci_attn_cached(ctx, rounded(q, dtype).cuda(), cache, dev(indptr), dev(src.ravel()), out, 1.0, lse=lse)
        ctx.sync()
        # with 16 bits a weight of two parts may be off by 2^-18 more
        off = 32 * ref.U if dtype == "fp32" else 32 * ref.U + 2.0 ** -18
        check(out, lse, want[:3] + (off * np.abs(want[0]),) + want[4:], n, dtype)


@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 1, 64, "fp32"), (8, 1, 128, "bf16"), (3, 1, 256, "fp16"), (16, 2, 64, "fp32")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_left_out_entries_of_shared_key_heads_may_hold_anything(heads, kv, dim, dtype, accumulate):
    """Slots that only left-out entries stand beside, slot 0 among them, hold codes of no number; the result is that of a cache with zeros there."""
    import paper_2503_01281_amd as dci
    from tests.test_gpu_attention import make_cache
    ctx = dci.Context(0)
    rng = np.random.default_rng(dim + heads)
    n_slots, sources, lengths = 90, 60, [70, 300, 0, 129, 66, 1000]
    cache, _ = make_cache(dci, n_slots, kv, dim, 16, rng)
    slots = (rng.permutation(n_slots - 20)[:sources] + 20).astype(np.int32)  # slots 0 .. 19 are named by nobody
    slots[rng.random(sources) < 0.3] = -1
    indptr, src = lists(lengths, sources, rng, outside=0.1)
    q = torch.randn(len(lengths), heads, dim, device="cuda").to(TYPES[dtype])
    before, got = cache.weight.clone(), []
    for code in (0, 0x7F, 0xFF):
        cache.codes[:20] = code
        cache.codes[20:][~torch.isin(torch.arange(20, n_slots, device="cuda"), dev(slots))] = code
        cache.weight.copy_(before)
        out, lse = torch.empty_like(q), torch.empty(len(lengths), heads, device="cuda")
        dci.dci_attn_cached(ctx, q, cache, dev(indptr), dev(src), out, 0.1, slots=dev(slots), lse=lse, accumulate=accumulate)
        ctx.sync()
        got.append((out, lse, cache.weight.clone()))
    assert torch.isfinite(got[0][0].float()).all()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_a_call_that_needs_no_workspace_is_taken_without_one():
    import ctypes as C

    import paper_2503_01281_amd as dci
    from paper_2503_01281_amd import binding as b
    ctx = dci.Context(0)
    cache = dci.KvCache(ctx, 32, 2, 32)
    q, out = torch.zeros(4, 2, 32, device="cuda"), torch.zeros(4, 2, 32, device="cuda")
    indptr, src = torch.zeros(5, dtype=torch.int64, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    for edges in (8, 64):
        a = b._attn_args(q, 2, 0, indptr, src[:edges], out, 1.0, None, None, None, 0)
        for accumulate in (0, 1):
            assert ctx.lib.dci_attn_workspace_bytes(C.byref(a), accumulate) == 0
            assert ctx.lib.dci_attn_cached(ctx.handle, C.byref(a), C.byref(cache.c), None, accumulate) == 0
    ctx.sync()
