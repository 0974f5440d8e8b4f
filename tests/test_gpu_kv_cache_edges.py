"""The 8-bit key/value cache where its launches end: more rows and heads than one launch has lanes for, entries without
rows.  Codes and scales are defined to the bit."""
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
