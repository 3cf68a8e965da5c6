"""The entry points over caches that are read in full, on a host without a GPU:
what they refuse before any HIP call (fake pointers are never dereferenced), the
workspace sizes, the binding's checks, and the oracle on cases done by hand."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from oracle import dense_oracle

FAKE = ctypes.c_void_p(0x7000_0000_0000)      # 16-byte aligned, never dereferenced
ODD = ctypes.c_void_p(0x7000_0000_0008)       # 8-byte aligned only
ODD4 = ctypes.c_void_p(0x7000_0000_0002)
OPS = range(5)


@pytest.fixture(scope="module")
def lib():
    return spec.load_library()


def dims(**kw):
    base = dict(B=2, L_cap=4096, n_layers=2, H_q=32, H_kv=8, T=64, window=1024, n_sink=4,
                P_cap=2048, n_sets=8, n_recent=32)
    base.update(kw)
    return spec.DenseDims.make(**base)


def size(lib, d, op):
    n = ctypes.c_size_t(0)
    return lib.spec_dense_workspace_size(ctypes.byref(d), op, ctypes.byref(n)), n.value


@pytest.mark.parametrize("field,value,status,ops", [
    ("B", 0, 1, OPS), ("L_cap", -1, 1, OPS), ("n_layers", 0, 1, OPS), ("H_kv", 0, 1, OPS),
    ("d", 0, 1, OPS), ("d", 64, 2, OPS), ("reserved", 1, 1, OPS), ("B", 70000, 2, OPS),
    ("kv_stride_b", 8, 1, OPS),                    # smaller than a sequence's block
    ("kv_stride_b", 4096 * 8 * 128 + 4, 1, OPS),   # not a multiple of 8
    ("kv_stride_layer", -8, 1, OPS), ("scale", -1.0, 1, OPS), ("scale", math.nan, 1, OPS),
    ("H_q", 30, 1, range(4)), ("H_q", 0, 1, range(4)), ("H_q", 8 * 129, 2, range(4)),
    ("window", 0, 1, (0, 1)), ("window", -5, 1, (0, 1)), ("n_sink", -1, 1, (0, 1, 4)),
    ("T", 0, 1, (1,)), ("T", -1, 1, (1, 4)), ("T", 1 << 22, 2, (1,)),
    ("P_cap", 0, 1, (2,)), ("prefix_stride_layer", 8, 1, (2,)),
    ("n_sets", 4, 2, (3, 4)), ("n_sets", 0, 2, (3, 4)), ("n_recent", -1, 1, (4,)),
    ("L_cap", 2 ** 31 - 1, 2, OPS),
])
def test_dims_validation(lib, field, value, status, ops):
    for op in OPS:
        d = dims()
        setattr(d, field, value)
        want = status if op in ops else 0
        assert size(lib, d, op)[0] == want, (field, op)


def test_any_number_of_query_heads(lib):
    for H_q in (8, 24, 40, 56, 8 * 17, 8 * 71, 8 * 128):
        for op in range(4):
            assert size(lib, dims(H_q=H_q), op)[0] == 0


def test_workspace_sizes(lib):
    assert lib.spec_dense_workspace_size(ctypes.byref(dims()), 0, None) == 1
    assert size(lib, dims(), 5)[0] == 1 and size(lib, dims(), -1)[0] == 1
    assert lib.spec_dense_workspace_size(None, 0, ctypes.byref(ctypes.c_size_t())) == 1
    # the logits of the accumulating attention, the lists of an eviction
    assert size(lib, dims(), spec.DENSE_ACCUM_DECODE)[1] >= 2 * 2 * 32 * 4096 * 4
    assert size(lib, dims(), spec.DENSE_EVICT)[1] >= 2 * 2 * 2 * 8 * 4096 * 4
    # the prefix's partial results: every query row at least once
    assert size(lib, dims(), spec.DENSE_PREFIX_DECODE)[1] >= 2 * 2 * 32 * 128 * 4


def calls(lib, d, ws, nws, **bad):
    """Every entry point with one argument replaced; yields (name, status)."""
    b = ctypes.byref
    a = dict(q=FAKE, k=FAKE, v=FAKE, lens=FAKE, q_lens=FAKE, out=FAKE, lse=FAKE, kp=FAKE, vp=FAKE,
             plen=FAKE, weights=FAKE, tokens=FAKE, counts=FAKE, keep=FAKE, pos=FAKE, kn=FAKE,
             vn=FAKE, nn=FAKE)
    a.update(bad)
    val = lambda p: None if p is None else p.value   # noqa: E731
    c = spec.Bounded(val(a["k"]), val(a["v"]), val(a["weights"]), val(a["tokens"]),
                     val(a["counts"]))
    yield "window_decode", ("q", "k", "v", "lens", "out", "lse"), lambda: (
        lib.spec_window_decode_attn(b(d), a["q"], a["k"], a["v"], a["lens"], a["out"], a["lse"],
                                    ws, nws, None))
    yield "window", ("q", "k", "v", "lens", "q_lens", "out", "lse"), lambda: (
        lib.spec_window_attn(b(d), a["q"], a["k"], a["v"], a["lens"], a["q_lens"], a["out"],
                             a["lse"], ws, nws, None))
    yield "prefix", ("q", "k", "v", "lens", "out", "lse", "kp", "vp", "plen"), lambda: (
        lib.spec_prefix_decode_attn(b(d), a["q"], a["kp"], a["vp"], a["plen"], a["k"], a["v"],
                                    a["lens"], a["out"], a["lse"], ws, nws, None))
    yield "accum", ("q", "k", "v", "counts", "out", "lse", "weights"), lambda: (
        lib.spec_accum_decode_attn(b(d), a["q"], a["k"], a["v"], a["counts"], a["weights"],
                                   a["out"], a["lse"], ws, nws, None))
    yield "evict", ("k", "v", "weights", "tokens", "counts", "keep", "pos", "kn", "vn", "nn"), \
        lambda: lib.spec_evict(b(d), b(c), a["keep"], a["pos"], a["kn"], a["vn"], a["nn"], ws, nws,
                               None)


NULLABLE = {"lse", "q_lens", "plen", "nn"}
WIDE = {"q", "k", "v", "out", "kp", "vp", "kn", "vn"}      # 16-byte aligned


@pytest.mark.parametrize("name", ["q", "k", "v", "lens", "q_lens", "out", "lse", "kp", "vp", "plen",
                                  "weights", "tokens", "counts", "keep", "pos", "kn", "vn", "nn"])
def test_pointers_are_checked_before_hip(lib, name):
    d, huge = dims(), 1 << 40
    wrong = [ODD if name in WIDE else ODD4] + ([] if name in NULLABLE else [None])
    used = 0
    for p in wrong:
        for what, names, call in calls(lib, d, FAKE, huge, **{name: p}):
            if name in names:
                assert call() == 1, (what, name, p)
                used += 1
    assert used and lib.spec_last_hip_error() == 0


def test_workspaces_are_checked_before_hip(lib):
    d = dims(L_cap=16384, window=16384, T=2)    # windows long enough to be split
    for op, (what, _, call) in enumerate(calls(lib, d, FAKE, 15)):
        assert size(lib, d, op)[1] > 16, what
        assert call() == 3, what
    for what, _, call in calls(lib, d, None, 1 << 40):
        assert call() == 3, what
    for what, _, call in calls(lib, d, ODD, 1 << 40):
        assert call() == 1, what
    for op, (what, _, call) in enumerate(calls(lib, d, FAKE, size(lib, d, 0)[1])):
        if op != 0 and size(lib, d, op)[1] > size(lib, d, 0)[1]:
            assert call() == 3, what
    assert lib.spec_evict(ctypes.byref(d), None, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 40,
                          None) == 1
    assert lib.spec_last_hip_error() == 0


def test_bindings_refuse_host_tensors_and_wrong_types():
    bf = dict(dtype=torch.bfloat16)
    q, K = torch.zeros((1, 2, 8, 128), **bf), torch.zeros((1, 2, 16, 8, 128), **bf)
    lens = torch.zeros(2, dtype=torch.int32)
    w = torch.zeros((1, 2, 8, 16))
    for call in (lambda: spec.window_decode_attn(q, K, K, lens, 8),
                 lambda: spec.window_attn(q[:, :, None], K, K, lens, 8),
                 lambda: spec.prefix_decode_attn(q, K[:, 0], K[:, 0], K, K, lens),
                 lambda: spec.accum_decode_attn(q, K, K, lens, w),
                 lambda: spec.evict(K, K, w, w.int(), lens, lens, lens)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError):
        spec.window_decode_attn(q.float(), K, K, lens, 8)
    with pytest.raises(ValueError):
        spec.window_attn(q, K, K, lens, 8)       # no dimension of query tokens


# ------------------------------------------------------------------ the oracle, by hand

def test_oracle_visible_tokens():
    assert dense_oracle.visible(9, 3, 2) == [0, 1, 7, 8, 9]
    assert dense_oracle.visible(1, 3, 2) == [0, 1]
    assert dense_oracle.visible(0, 1, 0) == [0]
    assert dense_oracle.visible(-1, 5, 5) == []


def test_oracle_window_and_prefix_by_hand():
    # equal logits: the output is the mean of the visible rows
    v = np.arange(5.0)[:, None, None] * np.ones((5, 1, 2))
    k, q = np.zeros((5, 1, 2)), np.ones((2, 1, 2))
    out, lse, spread = dense_oracle.window_attention(q, k, v, 3, 2, 1, 1.0)
    assert np.allclose(out[:, 0, 0], [(0 + 2 + 3) / 3, (0 + 3 + 4) / 3])
    assert np.allclose(lse[:, 0], math.log(3)) and np.allclose(spread, out)
    o, z = dense_oracle.prefix_attention(q[0], k[:2], v[:2], k[2:], v[2:], 1.0)
    assert np.allclose(o, 2.0) and np.allclose(z, math.log(5))
    o, z = dense_oracle.prefix_attention(q[0], k[:0], v[:0], k[:0], v[:0], 1.0)
    assert not o.any() and z[0] == -math.inf


def test_oracle_accumulates_per_set():
    q, k, v = np.zeros((4, 2)), np.zeros((3, 2, 2)), np.ones((3, 2, 2))
    _, _, w = dense_oracle.accumulate(q, k, v, 2, 1.0)
    assert w.shape == (2, 3) and np.allclose(w, 2 / 3)
    _, _, w = dense_oracle.accumulate(q, k, v, 1, 1.0)
    assert np.allclose(w, 4 / 3)


def test_oracle_evict_by_hand():
    w, t = [5.0, 1.0, 3.0, 1.0, 4.0], [10, 11, 12, 13, 14]
    # one new row into a full cache of five: the least weight, of equal ones the higher slot
    assert dense_oracle.evict_plan(w, t, 5, 1, 5, 15, 0, 0) == (5, [(3, ("new", 0))])
    # token 13 is one of the last three
    assert dense_oracle.evict_plan(w, t, 5, 1, 5, 15, 3, 0) == (5, [(1, ("new", 0))])
    # token 11 is a sink, 13 is recent
    assert dense_oracle.evict_plan(w, t, 5, 1, 5, 15, 3, 12) == (5, [(2, ("new", 0))])
    # down to three: slots 0, 2, 4 stay, the last moves into slot 1
    assert dense_oracle.evict_plan(w, t, 5, 0, 3, 15, 0, 0) == (3, [(1, ("held", 4))])
    # room left: the new rows are appended
    assert dense_oracle.evict_plan(w, t, 5, 2, 9, 15, 0, 0) == (7, [(5, ("new", 0)),
                                                                   (6, ("new", 1))])
    # more new rows than the budget: the last of them
    assert dense_oracle.evict_plan(w, t, 5, 4, 2, 15, 0, 0) == (2, [(0, ("new", 2)),
                                                                   (1, ("new", 3))])


def test_sizes_beyond_a_launch_are_refused(lib):
    big = dict(B=65535, L_cap=64, n_layers=1, T=1, n_sets=1)
    for op, kw, want in (
            (0, dict(H_q=32, H_kv=32), 0), (0, dict(H_q=64, H_kv=64), 2),      # KV heads
            (1, dict(H_q=32, H_kv=8, T=33), 2), (1, dict(H_q=32, H_kv=8, T=2), 0),
            (0, dict(H_q=8 * 127, H_kv=8), 2), (0, dict(H_q=8 * 128, H_kv=8), 0),
            (0, dict(H_q=127, H_kv=1), 2), (2, dict(H_q=127, H_kv=1), 2),      # a prime: 127 groups
            (3, dict(H_q=127, H_kv=1), 2), (1, dict(H_q=127, H_kv=1), 0),
            (3, dict(H_q=8, H_kv=8, L_cap=1 << 14), 2), (3, dict(H_q=8, H_kv=8, L_cap=1 << 12), 0)):
        status, n = size(lib, dims(**{**big, **kw}), op)
        assert status == want, (op, kw, status)
