"""The 8-bit key/value cache where its launches end: more rows and heads than one launch has lanes for, entries without
rows, two errors at a time.  Codes and scales are defined to the bit."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import attention_reference as ref
from tests.test_gpu_kv_cache import compare, dev, held_by, some_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dim,dtype", [(128, 256, "fp16"), (128, 200, "fp32")])
def test_a_bound_of_more_rows_than_one_launch_writes(heads, dim, dtype):
    """Eight million rows of 128 heads, counted on the GPU: 128 wavefronts more than have their lanes counted in 32 bits, so that a launch of all of
    them would run those 128, 16 rows, and say nothing.  All but the first 37 rows are not there."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(dim)
    n_slots, n, bound = 70, 37, 2 ** 23 + 16
    cache = dci.KvCache(ctx, n_slots, heads, dim, 16)
    held, exponents = held_by(cache)
    slots = np.full(bound, -1, dtype=np.int32)
    slots[:n] = np.sort(rng.permutation(n_slots)[:n])
    k, v = some_rows(rng, n, heads, dim, dtype), some_rows(rng, n, heads, dim, dtype)
    at, kd, vd, n_dev = dev(slots), k.cuda(), v.cuda(), torch.tensor([n], dtype=torch.int64, device="cuda")
    ctx.check(ctx.lib.dci_kv_write(ctx.handle, C.byref(cache.c), at.data_ptr(), bound, n_dev.data_ptr(), {"fp32": dci.DCI_F32, "fp16": dci.DCI_F16}[dtype],
                                   kd.data_ptr(), heads * dim, vd.data_ptr(), heads * dim))
    ctx.sync()
    ref.write(held, exponents, slots[:n], k.double().numpy(), v.double().numpy(), n_slots, 16)
    compare(cache, held, exponents)


@pytest.mark.parametrize("n", [0, 1, 4, 15, 16, 17, 63, 64, 130])
@pytest.mark.parametrize("heads,dim,dtype,block", [(4, 64, "bf16", 16), (2, 128, "fp32", 64), (3, 41, "fp16", 8), (1, 7, "fp32", 1), (2, 256, "bf16", 32)])
def test_entries_outside_the_cache_need_no_rows(n, heads, dim, dtype, block):
    """Slots as admission leaves them: those that were given, -1 behind, and rows of keys and values only for the former."""
    import paper_2503_01281_amd as dci
    ctx = dci.Context(0)
    rng = np.random.default_rng(n + dim)
    n_slots, entries = 200, 190
    cache = dci.KvCache(ctx, n_slots, heads, dim, block)
    held, exponents = held_by(cache)
    slots = np.full(entries, -1, dtype=np.int32)
    slots[:n] = np.sort(rng.permutation(n_slots)[:n])
    k, v = some_rows(rng, n, heads, dim, dtype), some_rows(rng, n, heads, dim, dtype)
    kd, vd, at = k.cuda(), v.cuda(), dev(slots)
    p = [t.data_ptr() if n else at.data_ptr() for t in (kd, vd)]  # without rows: any address that is not null
    ctx.check(ctx.lib.dci_kv_write(ctx.handle, C.byref(cache.c), at.data_ptr(), entries, None, {"fp32": dci.DCI_F32, "bf16": dci.DCI_BF16, "fp16": dci.DCI_F16}[dtype],
                                   p[0], heads * dim, p[1], heads * dim))
    ctx.sync()
    ref.write(held, exponents, slots[:n], k.double().numpy(), v.double().numpy(), n_slots, block)
    compare(cache, held, exponents)


@pytest.mark.parametrize("order", [("batch", "write"), ("write", "batch"), ("batch",), ("write",)])
def test_a_voided_batch_and_bad_slots_are_both_reported(order, tiny):
    """Two errors between two waits: the one does not hide the other.  The batch is voided as by a wait that ends: tiles numbered from 1 wait for
    tile 0, 200 polls long."""
    import paper_2503_01281_amd as dci
    from tests import gpu_util as gu
    w, n = tiny["w"], 600
    ctx = dci.Context(0, workspace_bytes=64 << 20)
    graph = gu.make_graph(tiny["indptr"], tiny["indices"], tiny["feat"])
    blk = dci.Blocks(ctx, w.num_nodes, n, w.fanouts)
    cache = dci.KvCache(ctx, 64, 2, 32, 16)
    rows, seeds, bad = torch.ones(2, 2, 32, device="cuda"), gu.dev(tiny["seeds"][:n]), dev(np.array([6, 5], dtype=np.int32))
    ctx.set_option(dci.DCI_OPT_RELABEL_SPIN_LIMIT, 200)
    ctx.set_option(dci.DCI_OPT_TEST_RELABEL_FIRST_TICKET, 1)
    for what in order:
        if what == "batch":
            dci.dci_sample_khop(ctx, graph, None, seeds, 0, w.fanouts, w.rng_seed, blk)
        else:
            dci.dci_kv_write(ctx, cache, bad, rows, rows)
        torch.cuda.synchronize()
    with pytest.raises(dci.DciError) as e:
        ctx.sync()
    assert ("relabel scan timed out" in str(e.value) and "must not be used" in str(e.value)) == ("batch" in order)
    assert ("strictly ascending" in str(e.value)) == ("write" in order)
    assert e.value.code == (-3 if "batch" in order else -1)
    ctx.sync()  # reported once
