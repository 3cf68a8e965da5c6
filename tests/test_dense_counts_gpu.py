"""The entry points over caches that are read in full on inputs whose every output is known
exactly (dense_bounds): every layer, sequence, query and head is compared, so that a token
lost, doubled or taken from elsewhere shows, at the end of a tile, part or window as
anywhere.  Sizes for every plan: 32, 64, 128 and 256 rows with the tokens whole and in
parts, one, two and four column groups beside each other, logits in LDS and in memory."""
import math

import pytest
import torch

import paper_2512_00722_amd as spec
from tests import dense_bounds as db
from tests import test_dense_gpu as base
from tests import test_dense_sizes_gpu as sizes
from tests.dense_bounds import D, U
from tests.gpu_helpers import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def queries(shape, dev):
    g = torch.Generator(device=dev).manual_seed(7)
    return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)


def counted_cache(n, B, cap, H_kv, lens, dev):
    """Keys of zeros, counted values; NaN behind the lengths."""
    V = db.counted_values(n, B, cap, H_kv, dev)
    K = torch.zeros_like(V)
    for b, L in enumerate(lens):
        K[:, b, L:], V[:, b, L:] = math.nan, math.nan
    return K, V


def close(got, want, rel, what):
    """Within rel of want (-inf: equal)."""
    ok = ((got.double() - want).abs() <= rel * want.abs()) | (got.double() == want)
    assert bool(ok.all()), (what, int((~ok).sum()))


def close_heads(out, lse, want, n, layer, b, H_kv, rel, what):
    """out [..][H_q][D] and lse [..][H_q] of one layer and sequence against want [..][D] at
    shift 0 and n [..] tokens."""
    G = lse.shape[-1] // H_kv
    for g in range(H_kv):
        w = torch.roll(want, db.shift_of(layer, b, g), -1)[..., None, :]
        close(out[..., g * G:(g + 1) * G, :], w, rel, (what, "out", layer, b, g))
    close(lse, db.lse_of(n)[..., None], 6 * U, (what, "lse", layer, b))


# ------------------------------------------------------------------ decoding

DECODE = [c[:7] for c in base.WINDOW_DECODE] + [
    # layers, H_q, H_kv, cap, lens, window, sinks
    (8, 16, 4, 2100, [2100 - 97 * b for b in range(16)], 1000, 4),     # four groups, in parts
    (32, 32, 8, 1200, [1200, 1003, 1004, 1005, 0, 1, 777, 1199], 1000, 4),         # four groups
    (4, 6, 2, 700, [(b * 389) % 701 for b in range(64)], 600, 3),                  # two
    (1, 32, 8, 20011, [20011, 19999], 15000, 16),                                  # in many parts
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_l{c[3]}_w{c[5]}_s{c[6]}")
def test_window_decode(dev, case):
    n, H_q, H_kv, cap, lens, window, sinks = case
    announce(f"counted window decode {case}")
    K, V = counted_cache(n, len(lens), cap, H_kv, lens, dev)
    q = queries((n, len(lens), H_q, D), dev)
    out, lse = spec.window_decode_attn(q, K, V, i32(lens, dev), window, n_sink=sinks)
    table = db.counts_table(cap, dev)
    want, m = db.counted_window(table, torch.tensor(lens, device=dev) - 1, window, sinks)
    for layer in range(n):
        for b in range(len(lens)):
            close_heads(out[layer, b], lse[layer, b], want[b], m[b], layer, b, H_kv, 4 * U, case)


ACCUM = [(c[0], len(c[4]), c[1], c[2], c[3], c[5]) for c in base.ACCUM] + sizes.ACCUM


@pytest.mark.parametrize("case", ACCUM, ids=lambda c: f"n{c[0]}_b{c[1]}_h{c[2]}_{c[3]}_l{c[4]}_s{c[5]}")
def test_accum(dev, case):
    n, B, H_q, H_kv, cap, n_sets = case
    announce(f"counted accum {case}")
    counts = [cap if b == 0 else (b * 7919) % (cap + 1) for b in range(B)]
    K, V = counted_cache(n, B, cap, H_kv, counts, dev)
    q = queries((n, B, H_q, D), dev)
    g = torch.Generator(device=dev).manual_seed(8)
    w0 = torch.rand((n, B, n_sets, cap), generator=g, device=dev)
    w = w0.clone()
    out, lse = spec.accum_decode_attn(q, K, V, i32(counts, dev), w)
    table = db.counts_table(cap, dev)
    want, m = db.counted_window(table, torch.tensor(counts, device=dev) - 1, cap, 0)
    for layer in range(n):
        for b in range(B):
            c = counts[b]
            close_heads(out[layer, b], lse[layer, b], want[b], m[b], layer, b, H_kv, 4 * U, case)
            assert torch.equal(w[layer, b, :, c:], w0[layer, b, :, c:])
            # 2^-log2(n): the logarithm is off by 2 U of itself, and by 4 U more where it comes
            # by way of the log-sum-exp (two products, two constants), times ln 2 log2(n) in
            # the weight; the exponential by 2 U; H_q / n_sets are added, and their sum to the
            # old weight
            add = H_q // n_sets / max(c, 1)
            tol = (5 * math.log2(max(c, 2)) + 6 + H_q // n_sets) * U * add
            err = (w[layer, b, :, :c].double() - w0[layer, b, :, :c].double() - add).abs()
            assert bool((err <= tol + U * w[layer, b, :, :c].double()).all()), (layer, b)


# ------------------------------------------------------------------ chunks

WINDOW = [c for c in base.WINDOW] + [(1, *c) for c in sizes.WINDOW] + [
    # layers, H_q, H_kv, cap, T, lens, q_lens, window, sinks
    (1, 24, 8, 3751, 740, [3751, 3000, 741], [740, 739, 740], 3273, 4),       # 256 rows, window
    (1, 14, 2, 11143, 905, [11143], None, 10375, 4),                          # ... in parts
    (1, 64, 8, 11287, 77, [11287, 9000, 77], None, 7663, 4),                  # 128 rows in parts
    (1, 6, 2, 9021, 126, [9020], None, 4537, 5),                              # 64
    (1, 3, 1, 1449, 16, [1449], None, 910, 4),                                # 32
    (2, 32, 8, 2048, 2048, [2048, 2000], [2048, 2000], 1000, 4),
]


@pytest.mark.parametrize("case", WINDOW, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_l{c[3]}_t{c[4]}_w{c[7]}_s{c[8]}")
def test_window(dev, case):
    n, H_q, H_kv, cap, T, lens, q_lens, window, sinks = case
    announce(f"counted window {case}")
    B = len(lens)
    K, V = counted_cache(n, B, cap, H_kv, lens, dev)
    q = queries((n, B, T, H_q, D), dev)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:-1], 7.0, device=dev)
    spec.window_attn(q, K, V, i32(lens, dev), window, n_sink=sinks,
                     q_lens=None if q_lens is None else i32(q_lens, dev), out=out, lse=lse)
    table = db.counts_table(cap, dev)
    for b in range(B):
        r = T if q_lens is None else q_lens[b]
        p = torch.arange(lens[b] - r, lens[b], device=dev)
        want, m = db.counted_window(table, p, window, sinks)
        for layer in range(n):
            assert (out[layer, b, r:] == 7.0).all() and (lse[layer, b, r:] == 7.0).all()
            close_heads(out[layer, b, :r], lse[layer, b, :r], want, m, layer, b, H_kv,
                        2.0 ** -8 + 4 * U, case)


# ------------------------------------------------------------------ shared prefix

PREFIX = [c for c in base.PREFIX] + [(1, *c) for c in sizes.PREFIX] + [
    # layers, H_q, H_kv, P_cap, P, cap, lens
    (1, 32, 8, 20011, 20000, 777, [777, 0, 1, 300] * 8 + [776, 32]),         # 136 rows
    (2, 32, 8, 4000, 3999, 200, [200, 3] * 33),                              # 264: two row tiles
    (1, 4, 1, 32769, None, 33, [33] * 7),
]


@pytest.mark.parametrize("case", PREFIX, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_p{c[3]}_{c[4]}_b{len(c[6])}")
def test_prefix(dev, case):
    n, H_q, H_kv, P_cap, P, cap, lens = case
    announce(f"counted prefix {case}")
    B, rows = len(lens), P_cap if P is None else P
    K, V = counted_cache(n, B, cap, H_kv, lens, dev)
    Kp, Vp = (t[:, 0] for t in counted_cache(n, 1, P_cap, H_kv, [rows], dev))
    q = queries((n, B, H_q, D), dev)
    out, lse = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32(lens, dev),
                                       prefix_len=None if P is None else i32([P], dev))
    own, pre = db.counts_table(cap, dev), db.counts_table(P_cap, dev)[rows]
    for b, L in enumerate(lens):
        m = torch.tensor(rows + L, device=dev)
        for layer in range(n):
            # the prefix has the shifts of sequence 0: its sums are moved back by b's
            both = torch.roll(pre, db.shift_of(layer, 0, 0) - db.shift_of(layer, b, 0), 0) + own[L]
            close_heads(out[layer, b], lse[layer, b], both / m.clamp(min=1), m, layer, b, H_kv,
                        4 * U, case)
