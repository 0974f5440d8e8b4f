"""What of the attention calls and the key/value cache needs no GPU: sizes, refusals without a context, and the reference that the GPU tests
are held to against closed forms."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from tests import attention_reference as ref


@pytest.fixture(scope="module")
def lib():
    import paper_2503_01281_amd as dci
    return dci.load_library()


def test_calls_without_a_context_are_refused(lib):
    from paper_2503_01281_amd import binding as b
    a, c = b._Attn(), b._KvCache()
    assert lib.dci_attn_forward(None, C.byref(a), None, 0, None, 0) == -1
    assert lib.dci_attn_cached(None, C.byref(a), C.byref(c), None, 0) == -1
    assert lib.dci_kv_clear(None, C.byref(c)) == -1
    assert lib.dci_kv_write(None, C.byref(c), None, 0, None, 0, None, 0, None, 0) == -1
    assert lib.dci_kv_read(None, C.byref(c), None, 0, None, 0, None, 0, None, 0) == -1
    assert lib.dci_kv_admit(None, C.byref(c), None, 0, None, 0, None, None, None, None, None) == -1


def test_workspace_sizes(lib):
    from paper_2503_01281_amd import binding as b

    def need(accumulate=0, **kw):
        a = b._Attn(n_rows=100, n_edges=1500, n_src=10, max_list=15, n_heads=4, kv_heads=4, head_dim=64)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.dci_attn_workspace_bytes(C.byref(a), accumulate)

    up = lambda x: -(-x // 256) * 256
    assert need() == need(1) == 0                          # short lists need none
    chunks = -(-1500 // 16)  # few entries: the shortest chunks
    parts = up(chunks * 2 * 4 * 2 * 4) + up(chunks * 2 * 4 * 64 * 4)
    assert need(max_list=0) == need(max_list=65) == parts  # lists that may be longer than 64
    assert need(1, max_list=0) == parts + up(1500 * 4 * 4) + up(100 * 4 * 4)  # a score per entry and head, a sum per row and head
    assert need(n_edges=0, max_list=0) == 0
    for bad in (dict(n_rows=-1), dict(n_heads=3), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=300), dict(n_edges=2 ** 40)):
        assert need(1, **bad) == 0
    assert lib.dci_attn_workspace_bytes(None, 0) == 0
    assert 0 < lib.dci_kv_admit_workspace_bytes(1, 0) < lib.dci_kv_admit_workspace_bytes(10 ** 6, 10 ** 5)
    assert lib.dci_kv_admit_workspace_bytes(0, 10) == 0 and lib.dci_kv_admit_workspace_bytes(10, -1) == 0


def test_the_reference_rounds_as_torch_does():
    x = torch.linspace(-460, 460, 40001).double()
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.to_e4m3(x.numpy()), want)
    small = torch.linspace(-0.05, 0.05, 20001).double()
    assert np.array_equal(ref.to_e4m3(small.numpy()), small.to(torch.float8_e4m3fn).double().numpy())
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(ref.e4m3_values(), nan=1e9), np.nan_to_num(every, nan=1e9))
    for amax in (448.0, 449.0, 224.0, 1e-3, 3.4e38, 1e-45):
        e = ref.need_exponent(amax)
        assert (448.0 * 2.0 ** e >= amax or e == 119) and (448.0 * 2.0 ** (e - 1) < amax or e == -100)


def test_the_reference_attends_as_a_softmax_does():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((m, 4, 8)) for m in (3, 6, 6))
    indptr, where = [0, 2, 2, 7], np.array([0, 5, 1, 1, -1, 2, 3])
    bias = rng.standard_normal((7, 1))
    bias[3] = -math.inf
    out, lse, p, out_err, lse_err, p_err = ref.attend(q, k, v, indptr, where, 0.5, bias)
    assert (out[1] == 0).all() and np.isneginf(lse[1]).all() and (p[3] == 0).all() and (p[4] == 0).all()
    for i, e in ((0, [0, 1]), (2, [2, 5, 6])):
        for h in range(4):
            z = torch.from_numpy(k[where[e], h] @ q[i, h] * 0.5 + bias[e, 0])
            w = torch.softmax(z, 0).numpy()
            assert np.allclose(out[i, h], w @ v[where[e], h], rtol=0, atol=1e-14) and np.allclose(p[e, h], w, atol=1e-15)
            assert abs(float(torch.logsumexp(z, 0)) - lse[i, h]) < 1e-14
    assert 0 < out_err[0].max() < 1e-5 and 0 < lse_err[0].max() < 1e-5 and 0 < p_err.max() < 1e-5


def test_the_reference_writes_and_admits():
    held, exponents = np.zeros((4, 2, 1, 2)), np.full((2, 2, 1), -1000.0)
    ref.write(held, exponents, [0], np.array([[[448.0, 1.0]]]), np.array([[[0.0, 0.0]]]), 4, 2)
    assert exponents[0, 0, 0] == 0 and exponents[0, 1, 0] == -100 and held[0, 0, 0].tolist() == [448.0, 1.0]
    ref.write(held, exponents, [1], np.array([[[900.0, 2.0]]]), np.array([[[1.0, 0.0]]]), 4, 2)  # the scale grows, slot 0 is rounded anew
    assert exponents[0, 0, 0] == 2 and held[0, 0, 0].tolist() == [112.0, 0.25] and held[1, 0, 0].tolist() == [224.0, 0.5]
    remap, node, weight = np.array([0, -1, 1, -1]), np.array([0, 2]), np.array([5, 3])
    slots, fresh, fresh_slots, counts = ref.admit(remap, node, weight, np.array([3, 0, 3, 1]))
    assert slots.tolist() == [1, 0, 1, -1] and fresh.tolist() == [0, -1, -1, -1] and fresh_slots.tolist() == [1, -1, -1, -1]
    assert counts.tolist() == [1, 2, 1, 1] and remap.tolist() == [0, -1, -1, 1] and node.tolist() == [0, 3] and weight.tolist() == [5, 1]


@pytest.mark.parametrize("heads,kv,dim", [(128, 128, 16), (128, 1, 64), (32, 8, 128), (4, 4, 64), (1, 1, 1)])
@pytest.mark.parametrize("edges", [10 ** 6, 67_225_600, 2 ** 28 + 1, 10 ** 9, 2 ** 33 + 7, 2 ** 38])
def test_no_launch_has_more_lanes_than_32_bits_count(lib, heads, kv, dim, edges):
    """The pieces of long lists, two to a chunk and head, are joined by a workgroup of 256 lanes to a chunk and head."""
    from paper_2503_01281_amd import binding as b
    a = b._Attn(n_rows=2 ** 31 - 1, n_edges=edges, n_src=10, max_list=0, n_heads=heads, kv_heads=kv, head_dim=dim)
    piece = 2 * 4 + -(-dim // 16) * 16 * 4
    chunks = (lib.dci_attn_workspace_bytes(C.byref(a), 0) - 2 * 255) // (2 * heads * piece)  # of two arrays on whole 256 bytes
    assert 0 < chunks * heads * 256 < 2 ** 32
    assert chunks * 2 ** 22 >= edges  # and a chunk stays one that a wavefront goes through in milliseconds


@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 4, 64, 0), (16, 4, 64, 1), (32, 8, 128, 1), (128, 128, 16, 2), (1, 1, 1, 0), (8, 4, 128, 2), (128, 1, 256, 0)])
@pytest.mark.parametrize("bias", [0, 1])
def test_the_workspace_of_a_call_does_for_every_smaller_one(lib, heads, kv, dim, dtype, bias):
    from paper_2503_01281_amd import binding as b

    def need(edges, rows, max_list, accumulate):
        a = b._Attn(n_rows=rows, n_edges=edges, n_src=10, max_list=max_list, n_heads=heads, kv_heads=kv, head_dim=dim, dtype=dtype,
                    bias=64 if bias else None, bias_heads=bias)
        return lib.dci_attn_workspace_bytes(C.byref(a), accumulate)

    rng = np.random.default_rng(heads + dim)
    # both sides of every place where chunks get longer, and sizes between
    sizes = {0, 1, 64, 65, 2 ** 38} | {int(2 ** x) for x in rng.uniform(6, 38, 200)}
    for chunk in (16, 32, 64, 128, 256, 512, 1024, 4096):
        for waves in (1, 2, 3, 4, 8, 16, 32, 64, 128):
            sizes |= {chunk * (wanted // waves + 1) + d for wanted in (1024, 4096) for d in (-1, 0, 1)}
        sizes |= {min(2 ** 38, chunk * ((2 ** 24 - 1) // heads) + d) for d in (0, 1)}
    for accumulate in (0, 1):
        for max_list in (0, 64, 65, 1000):
            needs = [need(e, 1000, max_list, accumulate) for e in sorted(sizes)]
            assert needs == sorted(needs)
        lists = [need(10 ** 6, 1000, m, accumulate) for m in (1, 64, 65, 10 ** 6, 2 * 10 ** 6, 0)]
        assert lists == sorted(lists)
        rows = [need(10 ** 6, r, 0, accumulate) for r in (0, 1, 999, 10 ** 6, 2 ** 31 - 1)]
        assert rows == sorted(rows)
