"""The entry points over caches that are read in full, against float64: window
attention (one token and chunks), a shared prefix, accumulated weights,
eviction, and runs of them together.

Tolerances.  With unit roundoff u = 2^-24 of fp32, a logit is a sum of d = 128
products of exact bf16 values: off by at most (d + 2) u sum |q k| scale, and its
power of two by another 2 u |logit|.  `delta` is the sum of the two, taken for
the largest |q| |k| of the case.  A weight is then off by 2 delta + 2^-17
relatively where it enters the sums as a bf16 pair, and by 2^-8 (half a step)
more where it is rounded to bf16; sums of up to n terms add n u at most.  An
output is off by that times sum p |v|, and by 2^-8 of itself where it is bf16.
"""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from oracle import dense_oracle
from tests.gpu_helpers import announce, f64, need_gpu

pytestmark = pytest.mark.gpu

D = 128
SCALE = 1.0 / math.sqrt(D)
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


def normal(shape, seed, dev, sd=1.0):
    g = torch.Generator().manual_seed(seed)
    return (sd * torch.randn(shape, generator=g)).to(torch.bfloat16).to(dev)


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def delta(q, k, scale=SCALE):
    """Error of a logit plus that of its exponential's argument (see above)."""
    if q.size == 0 or k.size == 0:
        return 0.0
    top = np.abs(q).reshape(-1, D).max(0) @ np.abs(k).reshape(-1, D).max(0) * scale
    return (D + 2) * U * top + 2 * U * 1.5 * top


def weight_error(q, k, n, scale=SCALE):
    return 2 * delta(q, k, scale) + 2.0 ** -17 + n * U


def finite(x):
    return np.where(np.isfinite(x), x, 0.0)


def check(got, want, tol, what):
    got = np.asarray(got, dtype=np.float64)
    same = np.isinf(want) & (got == want)
    err = np.where(same, 0.0, np.abs(got - np.where(same, 0.0, want)))
    assert np.isfinite(err).all(), what
    bad = err > tol
    assert not bad.any(), (what, float(err.max()), float((err / np.maximum(tol, 1e-300)).max()))


def cache(n, B, cap, H_kv, seed, dev, lens=None, lo=None):
    """K and V; rows behind a sequence's length hold NaN."""
    K, V = (normal((n, B, cap, H_kv, D), seed + i, dev) for i in range(2))
    if lens is not None:
        for b, L in enumerate(lens):
            K[:, b, max(0, min(L, cap)):] = math.nan
            V[:, b, max(0, min(L, cap)):] = math.nan
    return K, V


# ------------------------------------------------------------------ window, one token

WINDOW_DECODE = [
    # layers, H_q, H_kv, cap, lens, window, sinks
    (1, 8, 8, 64, [64], 16, 4),
    (1, 32, 8, 300, [0, 1, 2, 5, 299, 300], 37, 4),
    (2, 28, 4, 700, [700, 333, 64, 0, 1], 128, 3),
    (1, 3, 1, 1000, [1000, 17], 5000, 0),
    (1, 24, 1, 515, [515, 100], 100, 16),       # 24 query heads on one KV head
    (1, 71, 1, 130, [130, 65], 64, 1),          # a prime number of them
    (3, 64, 8, 2100, [2100, 1500, 40], 1024, 4),
    (1, 16, 16, 40, [40], 1, 0),
    (1, 16, 16, 40, [40, 3], 1, 64),            # sinks cover the cache
    (32, 32, 8, 70, [70, 69, 3, 0, 70, 11, 64, 32, 33, 31], 33, 2),  # several units a wavefront
]


@pytest.mark.parametrize("case", WINDOW_DECODE, ids=lambda c: f"h{c[1]}_{c[2]}_w{c[5]}_s{c[6]}")
def test_window_decode(dev, case):
    n, H_q, H_kv, cap, lens, window, sinks = case
    announce(f"window decode {case}")
    B = len(lens)
    K, V = cache(n, B, cap, H_kv, 1, dev, lens)
    q = normal((n, B, H_q, D), 3, dev)
    # tokens that no query sees, inside the sequence, hold NaN as well
    for b, L in enumerate(lens):
        hidden = [t for t in range(L) if t not in set(dense_oracle.visible(L - 1, window, sinks))]
        K[:, b, hidden] = math.nan
        V[:, b, hidden] = math.nan
    out, lse = spec.window_decode_attn(q, K, V, i32(lens, dev), window, n_sink=sinks)
    torch.cuda.synchronize()
    for l, b in itertools.product(range(min(n, 3)), range(B)):
        l = l if n < 4 else l * (n - 1) // 2
        qq, kk, vv = f64(q[l, b]), f64(K[l, b]), f64(V[l, b])
        want, wlse, spread = dense_oracle.window_attention(qq[None], kk, vv, lens[b] - 1, window,
                                                           sinks, SCALE)
        e = weight_error(qq, finite(kk), cap)
        check(out[l, b].cpu(), want[0], e * spread[0] * 2 + 1e-30, ("out", l, b))
        check(lse[l, b].cpu(), wlse[0], e + 16 * U * np.abs(finite(wlse[0])), ("lse", l, b))


def test_window_decode_strided(dev):
    """Caches that are parts of larger ones, layers and sequences apart."""
    big_k, big_v = (normal((3, 4, 200, 4, D), 11 + i, dev) for i in range(2))
    K, V = big_k[::2, ::2, :150], big_v[::2, ::2, :150]
    q = normal((2, 2, 16, D), 13, dev)
    lens = i32([150, 77], dev)
    got = spec.window_decode_attn(q, K, V, lens, 40, n_sink=2)
    want = spec.window_decode_attn(q, K.contiguous(), V.contiguous(), lens, 40, n_sink=2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_window_decode_agrees_with_the_selection(dev):
    """A window without sinks over fewer tokens than it holds is the compact sparse
    attention: each is off by at most its own error."""
    K, V = cache(2, 3, 256, 8, 21, dev)
    q = normal((2, 3, 32, D), 23, dev)
    lens = i32([256, 100, 1], dev)
    a = spec.window_decode_attn(q, K, V, lens, 256)
    b = spec.sparse_decode_attn(q, K, V, lens)
    e = weight_error(f64(q), f64(K), 256)
    assert (a[0] - b[0]).abs().max() <= 4 * e * float(V.abs().max())
    assert (a[1] - b[1]).abs().max() <= 2 * e + 32 * U * float(b[1].abs().max())


# ------------------------------------------------------------------ window, chunks

WINDOW = [
    # layers, H_q, H_kv, cap, T, lens, q_lens, window, sinks
    (1, 4, 4, 64, 1, [64], None, 16, 2),
    (1, 32, 8, 100, 2, [100, 1, 0], None, 30, 4),        # positions below 0 see nothing
    (1, 28, 4, 300, 17, [300, 17, 9, 40], [17, 17, 9, 0], 50, 3),
    (2, 8, 2, 200, 33, [200, 150], [33, 5], 20, 0),
    (1, 3, 1, 400, 100, [400, 399], None, 77, 5),
    (1, 32, 2, 150, 70, [150, 90], [64, 70], 1, 1),      # only itself and a sink
    (1, 16, 1, 700, 9, [700], None, 1000, 0),            # few rows: the tokens are split
    (1, 8, 8, 1100, 40, [1100, 800], [40, 39], 1100, 4),
    (1, 130, 2, 90, 12, [90], None, 64, 2),              # 65 query heads a KV head
    (1, 2, 1, 500, 260, [500, 260], [260, 260], 129, 130),  # more sinks than the window
    (1, 8, 1, 220, 37, [220], None, 64, 70),
]


@pytest.mark.parametrize("case", WINDOW, ids=lambda c: f"h{c[1]}_{c[2]}_t{c[4]}_w{c[7]}_s{c[8]}")
def test_window(dev, case):
    n, H_q, H_kv, cap, T, lens, q_lens, window, sinks = case
    announce(f"window {case}")
    B = len(lens)
    K, V = cache(n, B, cap, H_kv, 31, dev, lens)
    q = normal((n, B, T, H_q, D), 33, dev)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:-1], 7.0, device=dev)
    spec.window_attn(q, K, V, i32(lens, dev), window, n_sink=sinks,
                     q_lens=None if q_lens is None else i32(q_lens, dev), out=out, lse=lse)
    torch.cuda.synchronize()
    rows = [T] * B if q_lens is None else q_lens
    for l, b in itertools.product(range(n), range(B)):
        r = rows[b]
        qq, kk, vv = f64(q[l, b, :r]), f64(K[l, b]), f64(V[l, b])
        want, wlse, spread = dense_oracle.window_attention(qq, kk, vv, lens[b] - r, window, sinks,
                                                           SCALE)
        e = weight_error(qq, finite(kk), cap)
        tol = (2 * e + 2.0 ** -8) * spread + 2.0 ** -8 * np.abs(want) + 1e-30
        check(f64(out[l, b, :r]), want, tol, ("out", l, b))
        check(lse[l, b, :r].cpu(), wlse, e + 16 * U * np.abs(finite(wlse)), ("lse", l, b))
        assert (out[l, b, r:] == 7.0).all() and (lse[l, b, r:] == 7.0).all()


@pytest.mark.parametrize("T,G", [(5, 1), (40, 4), (70, 8)])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_window_odd_values_reach_only_those_that_see_them(dev, T, G, odd):
    """A row of V with an infinity or a NaN in one dimension: the queries that see
    it have that value there, the others and the other dimensions are as if it
    were 0."""
    cap, window, sinks = 200, 30, 2
    K, V = cache(1, 1, cap, 1, 41, dev)
    q = normal((1, 1, T, G, D), 43, dev)
    bad = {cap - T // 2: 5, cap - T - 10: 64, cap - 1: 127, cap - window - T // 2: 33}
    clean = V.clone()
    for t, dim in bad.items():
        V[0, 0, t, 0, dim] = odd
        clean[0, 0, t, 0, dim] = 0.0
    got, _ = spec.window_attn(q, K, V, i32([cap], dev), window, n_sink=sinks)
    qq, kk, vv = f64(q[0, 0]), f64(K[0, 0]), f64(clean[0, 0])
    want, _, spread = dense_oracle.window_attention(qq, kk, vv, cap - T, window, sinks, SCALE)
    tol = (2 * weight_error(qq, kk, cap) + 2.0 ** -8) * spread + 2.0 ** -8 * np.abs(want) + 1e-30
    got = f64(got[0, 0])
    for i in range(T):
        seen = set(dense_oracle.visible(cap - T + i, window, sinks))
        for t, dim in bad.items():
            if t in seen:
                assert (np.isnan(got[i, :, dim]) if odd != odd else got[i, :, dim] == odd).all()
                got[i, :, dim] = want[i, :, dim]
    check(got, want, tol, "the other values")


def test_window_odd_keys(dev):
    """Keys that no query sees may hold anything; a key of NaN makes the outputs of
    those that see it NaN and no other."""
    T, cap, window = 50, 180, 20
    K, V = cache(1, 1, cap, 2, 51, dev)
    q = normal((1, 1, T, 8, D), 53, dev)
    K[0, 0, 150] = math.nan
    K[0, 0, :cap - T - window] = math.inf
    V[0, 0, :cap - T - window] = math.nan
    got, lse = spec.window_attn(q, K, V, i32([cap], dev), window)
    for i in range(T):
        sees = 150 in dense_oracle.visible(cap - T + i, window, 0)
        assert bool(torch.isnan(got[0, 0, i]).all()) == sees, i
        assert bool(torch.isfinite(got[0, 0, i]).all()) != sees, i


def test_window_chunks_and_single_tokens_agree(dev):
    """The decode entry point, and chunks of several lengths, on the same tokens."""
    n, B, H_q, H_kv, cap, window, sinks = 1, 2, 32, 8, 600, 100, 4
    K, V = cache(n, B, cap, H_kv, 61, dev)
    q = normal((n, B, 64, H_q, D), 63, dev)
    lens = i32([600, 333], dev)
    whole, wl = spec.window_attn(q, K, V, lens, window, n_sink=sinks)
    # each lse is off by at most delta; each output by 2^-8 of itself and of sum p |v|
    # (over 100 tokens or more: both well below 1)
    tol = 2 * delta(f64(q), f64(K))
    for first, T in ((0, 16), (16, 47), (63, 1)):
        part, pl = spec.window_attn(q[:, :, first:first + T].contiguous(), K, V,
                                    lens - (64 - first - T), window, n_sink=sinks)
        assert (part.float() - whole[:, :, first:first + T].float()).abs().max() <= 2.0 ** -5
        assert (pl - wl[:, :, first:first + T]).abs().max() <= tol
    one, ol = spec.window_decode_attn(q[:, :, 63].contiguous(), K, V, lens, window, n_sink=sinks)
    assert (one - whole[:, :, 63].float()).abs().max() <= 2.0 ** -5
    assert (ol - wl[:, :, 63]).abs().max() <= tol


# ------------------------------------------------------------------ shared prefix

PREFIX = [
    # layers, H_q, H_kv, P_cap, P (None: P_cap), cap, lens
    (1, 8, 8, 1, None, 1, [0, 1]),
    (1, 32, 8, 64, None, 40, [0, 40, 17]),
    (1, 32, 8, 1000, 999, 128, [128, 0, 1, 64]),
    (2, 28, 4, 333, 65, 50, [50, 3, 0, 7, 31]),
    (1, 16, 1, 700, 0, 30, [0, 30]),                      # no prefix yet
    (1, 6, 2, 2000, None, 600, [600] * 12 + [5]),
    (1, 64, 8, 515, None, 70, [70, 0, 9] * 7),            # 168 rows
    (1, 48, 1, 300, 257, 20, [20, 7]),
    (2, 128, 1, 130, None, 33, [33, 1, 0]),               # 384 rows
]


@pytest.mark.parametrize("case", PREFIX, ids=lambda c: f"h{c[1]}_{c[2]}_p{c[3]}_{c[4]}_b{len(c[6])}")
def test_prefix(dev, case):
    n, H_q, H_kv, P_cap, P, cap, lens = case
    announce(f"prefix {case}")
    B = len(lens)
    K, V = cache(n, B, cap, H_kv, 71, dev, lens)
    Kp, Vp = (normal((n, P_cap, H_kv, D), 73 + i, dev) for i in range(2))
    rows = P_cap if P is None else P
    Kp[:, rows:] = math.nan
    Vp[:, rows:] = math.nan
    q = normal((n, B, H_q, D), 75, dev)
    out, lse = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32(lens, dev),
                                       prefix_len=None if P is None else i32([P], dev))
    torch.cuda.synchronize()
    for l, b in itertools.product(range(n), range(B)):
        qq = f64(q[l, b])
        ks, vs = [f64(Kp[l, :rows]), f64(K[l, b, :lens[b]])], [f64(Vp[l, :rows]),
                                                               f64(V[l, b, :lens[b]])]
        want, wlse = dense_oracle.prefix_attention(qq, ks[0], vs[0], ks[1], vs[1], SCALE)
        spread, _ = dense_oracle.prefix_attention(qq, ks[0], np.abs(vs[0]), ks[1], np.abs(vs[1]),
                                                  SCALE)
        e = weight_error(qq, np.concatenate(ks), rows + cap)
        check(out[l, b].cpu(), want, 2 * e * spread + 1e-30, ("out", l, b))
        check(lse[l, b].cpu(), wlse, e + 16 * U * np.abs(finite(wlse)), ("lse", l, b))


def test_prefix_strided(dev):
    big = normal((3, 90, 4, D), 81, dev)
    Kp, Vp = big[::2, :70], normal((3, 90, 4, D), 82, dev)[::2, :70]
    big_k, big_v = (normal((3, 4, 60, 4, D), 83 + i, dev) for i in range(2))
    K, V = big_k[::2, 1:3, :50], big_v[::2, 1:3, :50]
    q = normal((2, 2, 8, D), 85, dev)
    lens = i32([50, 20], dev)
    got = spec.prefix_decode_attn(q, Kp, Vp, K, V, lens)
    want = spec.prefix_decode_attn(q, Kp.contiguous(), Vp.contiguous(), K.contiguous(),
                                   V.contiguous(), lens)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------------------------ accumulated weights

ACCUM = [
    # layers, H_q, H_kv, cap, counts, n_sets
    (1, 8, 8, 1, [1, 0], 8),
    (1, 32, 8, 70, [70, 1, 0, 33], 8),
    (2, 28, 4, 333, [333, 64, 5], 1),
    (1, 16, 1, 2000, [2000, 1999], 1),
    (1, 24, 2, 515, [515, 100], 2),
    (24, 32, 8, 61, [61, 30, 0, 7, 61, 60, 9, 32], 8),
]


@pytest.mark.parametrize("case", ACCUM, ids=lambda c: f"h{c[1]}_{c[2]}_l{c[3]}_s{c[5]}")
def test_accum(dev, case):
    n, H_q, H_kv, cap, counts, n_sets = case
    announce(f"accum {case}")
    B = len(counts)
    K, V = cache(n, B, cap, H_kv, 91, dev, counts)
    q = normal((n, B, H_q, D), 93, dev)
    w0 = torch.rand((n, B, n_sets, cap), generator=torch.Generator().manual_seed(94)).to(dev)
    w = w0.clone()
    out, lse = spec.accum_decode_attn(q, K, V, i32(counts, dev), w)
    w2 = w0.clone()
    out2, none = spec.accum_decode_attn(q, K, V, i32(counts, dev), w2, with_lse=False)
    assert none is None and torch.equal(out, out2) and torch.equal(w, w2)
    for l, b in itertools.product(range(n), range(B)):
        c = counts[b]
        qq, kk, vv = f64(q[l, b]), f64(K[l, b, :c]), f64(V[l, b, :c])
        want, wlse, add = dense_oracle.accumulate(qq, kk, vv, n_sets, SCALE)
        spread, _, _ = dense_oracle.accumulate(qq, kk, np.abs(vv), n_sets, SCALE)
        e = weight_error(qq, kk, cap)
        check(out[l, b].cpu(), want, 2 * e * spread + 1e-30, ("out", l, b))
        check(lse[l, b].cpu(), wlse, e + 16 * U * np.abs(finite(wlse)), ("lse", l, b))
        before = w0[l, b].double().cpu().numpy()
        check(w[l, b, :, :c].cpu(), before[:, :c] + add,
              (2 * e + 2.0 ** -19) * add + 2 * U * (before[:, :c] + add), ("weights", l, b))
        assert torch.equal(w[l, b, :, c:], w0[l, b, :, c:])


# ------------------------------------------------------------------ eviction

EVICT = [
    # layers, H_kv, per head, cap, counts, keep, T, n_new, recent, sinks
    (1, 2, True, 16, [16, 16], [16, 16], 1, None, 4, 2),
    (1, 4, False, 64, [64, 10, 0], [64, 64, 64], 5, [5, 0, 3], 8, 1),
    (2, 8, True, 100, [100, 37, 99], [50, 37, 100], 0, None, 10, 4),     # down to the budget
    (1, 1, True, 40, [40, 40, 40, 12], [20, 0, 1, 12], 30, [30, 30, 7, 30], 0, 0),
    (1, 2, False, 700, [700, 650], [600, 700], 90, None, 64, 4),
    (2, 2, True, 5000, [5000, 4100], [4096, 4099], 33, [33, 1], 100, 4),
    (1, 1, True, 20000, [20000, 17000], [9000, 16500], 7, None, 300, 4),  # keys beyond LDS
    (1, 2, True, 60, [60, 60], [60, 60], 3, None, 10 ** 9, 0),            # everything is recent
    (1, 2, True, 60, [60, 60], [30, 30], 4, None, 0, 10 ** 9),            # everything is a sink
]


def bounded(n, B, S, H_kv, cap, seed, dev):
    K, V = cache(n, B, cap, H_kv, seed, dev)
    r = np.random.default_rng(seed)
    w = r.exponential(1.0, (n, B, S, cap)).astype(np.float32)
    w[r.random(w.shape) < 0.3] = 0.25                     # many equal weights
    w[r.random(w.shape) < 0.05] = 0.0
    w[r.random(w.shape) < 0.02] = -0.0
    w[r.random(w.shape) < 0.02] = np.nan
    w[r.random(w.shape) < 0.01] = np.inf
    t = np.argsort(r.random((n, B, S, cap)), axis=-1).astype(np.int32)
    return K, V, torch.from_numpy(w).to(dev), torch.from_numpy(t).to(dev)


def evict_reference(x, S, counts, keep, pos, rows, k_new, v_new, recent, sinks):
    """The same, slot by slot, on copies; returns them and the counts."""
    K, V, w, t = (y.clone() for y in x)
    n, B, cap, H_kv, _ = K.shape
    per = H_kv // S
    wn, tn = w.cpu().numpy(), t.cpu().numpy()
    after = list(counts)
    for l, b, s in itertools.product(range(n), range(B), range(S)):
        after[b], moves = dense_oracle.evict_plan(wn[l, b, s], tn[l, b, s], counts[b], rows[b],
                                                  min(max(keep[b], 0), cap), pos[b], recent, sinks)
        heads = slice(s * per, (s + 1) * per)
        held = [(d, j) for d, (kind, j) in moves if kind == "held"]
        new = [(d, j) for d, (kind, j) in moves if kind == "new"]
        for pairs, ks, vs in ((held, x[0][l, b], x[1][l, b]),
                              (new, None if k_new is None else k_new[l, b],
                               None if v_new is None else v_new[l, b])):
            if pairs:
                d, j = (torch.tensor(y, device=K.device) for y in zip(*pairs))
                K[l, b, d, heads] = ks[j, heads]
                V[l, b, d, heads] = vs[j, heads]
        for d, j in held:
            w[l, b, s, d], t[l, b, s, d] = x[2][l, b, s, j], x[3][l, b, s, j]
        if new:
            d, j = (torch.tensor(y, device=K.device) for y in zip(*new))
            w[l, b, s, d] = 0.0
            t[l, b, s, d] = (pos[b] + j).to(torch.int32)
    return K, V, w, t, after


def same_bits(a, b):
    if a.dtype == torch.float32:
        a, b = a.view(torch.int32), b.view(torch.int32)
    elif a.dtype == torch.bfloat16:
        a, b = a.view(torch.int16), b.view(torch.int16)
    return torch.equal(a, b)


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"h{c[1]}_{c[2]}_l{c[3]}_t{c[6]}_r{c[8]}_s{c[9]}")
def test_evict(dev, case):
    n, H_kv, per_head, cap, counts, keep, T, n_new, recent, sinks = case
    announce(f"evict {case}")
    B, S = len(counts), H_kv if per_head else 1
    x = bounded(n, B, S, H_kv, cap, 101, dev)
    k_new = v_new = None
    if T:
        k_new, v_new = (normal((n, B, T, H_kv, D), 103 + i, dev) for i in range(2))
    pos = [cap + 3 * b for b in range(B)]
    rows = [T] * B if n_new is None else n_new
    K, V, w, t, after = evict_reference(x, S, counts, keep, pos, rows, k_new, v_new,
                                        min(recent, 10 ** 9), sinks)
    c = i32(counts, dev)
    spec.evict(*x, c, i32(keep, dev), i32(pos, dev), k_new=k_new, v_new=v_new,
               n_new=None if n_new is None else i32(n_new, dev), n_recent=recent, n_sink=sinks)
    torch.cuda.synchronize()
    assert c.tolist() == after
    for got, want, nm in zip(x, (K, V, w, t), ("K", "V", "weights", "tokens")):
        assert same_bits(got, want), nm


def test_evict_strided(dev):
    n, B, H_kv, cap, T = 2, 2, 2, 50, 6
    x = bounded(n, B, H_kv, H_kv, cap, 111, dev)
    big_k, big_v = (torch.zeros((2 * n, 2 * B, cap + 9, H_kv, D), dtype=torch.bfloat16, device=dev)
                    for _ in range(2))
    Ks, Vs = big_k[::2, ::2, :cap], big_v[::2, ::2, :cap]
    Ks.copy_(x[0])
    Vs.copy_(x[1])
    k_new, v_new = (normal((n, B, T, H_kv, D), 113 + i, dev) for i in range(2))
    args = dict(k_new=k_new, v_new=v_new, n_recent=5, n_sink=1)
    w, t, c = x[2].clone(), x[3].clone(), i32([50, 47], dev)
    spec.evict(Ks, Vs, w, t, c, i32([50, 50], dev), i32([80, 90], dev), **args)
    c2 = i32([50, 47], dev)
    spec.evict(*x, c2, i32([50, 50], dev), i32([80, 90], dev), **args)
    assert same_bits(Ks.contiguous(), x[0]) and same_bits(Vs.contiguous(), x[1])
    assert same_bits(w, x[2]) and same_bits(t, x[3]) and torch.equal(c, c2)
    assert not big_k[1::2].any() and not big_k[:, 1::2].any() and not big_k[:, :, cap:].any()


# ------------------------------------------------------------------ together

def test_bounded_decode_loop(dev):
    """Twelve decode steps of a model over bounded caches: each step's row goes in,
    evicting where the cache is full, and the attention adds its weights.  The
    same in float64 from the caches' own contents."""
    n, B, H_q, H_kv, cap, recent, sinks = 2, 3, 8, 2, 40, 6, 2
    K, V = cache(n, B, cap, H_kv, 121, dev)
    K.zero_(), V.zero_()
    w = torch.zeros((n, B, H_kv, cap), device=dev)
    t = torch.zeros((n, B, H_kv, cap), dtype=torch.int32, device=dev)
    counts, keep, pos = i32([0] * B, dev), i32([cap, 30, 5], dev), i32([0] * B, dev)
    first = normal((2, n, B, 35, H_kv, D), 123, dev)
    spec.evict(K, V, w, t, counts, keep, pos, k_new=first[0], v_new=first[1], n_recent=recent,
               n_sink=sinks)
    pos += 35
    assert counts.tolist() == [35, 30, 5]
    for step in range(12):
        kv = normal((2, n, B, 1, H_kv, D), 130 + step, dev)
        before = [y.clone() for y in (K, V, w, t)]
        c0 = counts.tolist()
        spec.evict(K, V, w, t, counts, keep, pos, k_new=kv[0], v_new=kv[1], n_recent=recent,
                   n_sink=sinks)
        ref = evict_reference(before, H_kv, c0, keep.tolist(), pos.tolist(), [1] * B, kv[0], kv[1],
                              recent, sinks)
        for got, want in zip((K, V, w, t), ref):
            assert same_bits(got, want), step
        pos += 1
        w0 = w.clone()
        q = normal((n, B, H_q, D), 150 + step, dev)
        out, _ = spec.accum_decode_attn(q, K, V, counts, w)
        for l, b in itertools.product(range(n), range(B)):
            c = int(counts[b])
            qq, kk, vv = f64(q[l, b]), f64(K[l, b, :c]), f64(V[l, b, :c])
            want, _, add = dense_oracle.accumulate(qq, kk, vv, H_kv, SCALE)
            spread, _, _ = dense_oracle.accumulate(qq, kk, np.abs(vv), H_kv, SCALE)
            e = weight_error(qq, kk, cap)
            check(out[l, b].cpu(), want, 2 * e * spread, ("out", step, l, b))
            old = w0[l, b, :, :c].double().cpu().numpy()
            check(w[l, b, :, :c].cpu(), old + add, (2 * e + 2.0 ** -19) * add + 2 * U * (old + add),
                  ("weights", step, l, b))
    # every new token of the last `recent` is still held
    for l, b, g in itertools.product(range(n), range(B), range(H_kv)):
        held = set(t[l, b, g, :int(counts[b])].tolist())
        newest = int(pos[b])
        assert set(range(newest - min(recent, int(counts[b]) - sinks), newest)) <= held


def test_captured_steps_replay(dev):
    """A decode step of every entry point in one captured graph, replayed with the
    program's own work between: each replay equals the eager calls."""
    n, B, H_q, H_kv, cap, P = 2, 3, 16, 4, 300, 200
    K, V = cache(n, B, cap, H_kv, 161, dev)
    Kp, Vp = (normal((n, P, H_kv, D), 163 + i, dev) for i in range(2))
    q = normal((n, B, H_q, D), 165, dev)
    qc = normal((n, B, 9, H_q, D), 166, dev)
    kv = normal((2, n, B, 1, H_kv, D), 167, dev)
    lens, keep = i32([300, 120, 0], dev), i32([300, 300, 300], dev)
    state = dict(w=torch.rand((n, B, H_kv, cap), device=dev),
                 t=torch.arange(cap, dtype=torch.int32, device=dev).expand(n, B, H_kv, cap)
                 .contiguous(), counts=i32([300, 120, 0], dev), pos=i32([900, 120, 0], dev),
                 K=K.clone(), V=V.clone())
    outs = {}

    def dims(**kw):
        return spec.DenseDims.make(B=B, L_cap=cap, n_layers=n, H_q=H_q, H_kv=H_kv, **kw)

    ws = {op: torch.full((max(16, spec.dense_workspace_size(dims(**kw), op)),), 255,
                         dtype=torch.uint8, device=dev)
          for op, kw in ((spec.DENSE_WINDOW_DECODE, dict(window=64, n_sink=2)),
                         (spec.DENSE_WINDOW, dict(window=64, n_sink=2, T=9)),
                         (spec.DENSE_PREFIX_DECODE, dict(P_cap=P)),
                         (spec.DENSE_ACCUM_DECODE, dict(n_sets=H_kv)),
                         (spec.DENSE_EVICT, dict(T=1, n_sets=H_kv)))}

    def step(s, o):
        spec.evict(s["K"], s["V"], s["w"], s["t"], s["counts"], keep, s["pos"], k_new=kv[0],
                   v_new=kv[1], n_recent=16, n_sink=2, ws=ws[spec.DENSE_EVICT])
        s["pos"] += 1
        o["a"] = spec.accum_decode_attn(q, s["K"], s["V"], s["counts"], s["w"], out=o.get("ao"),
                                        lse=o.get("al"), ws=ws[spec.DENSE_ACCUM_DECODE])
        o["w"] = spec.window_decode_attn(q, s["K"], s["V"], s["counts"], 64, n_sink=2,
                                         out=o.get("wo"), lse=o.get("wl"),
                                         ws=ws[spec.DENSE_WINDOW_DECODE])
        o["c"] = spec.window_attn(qc, s["K"], s["V"], s["counts"], 64, n_sink=2, out=o.get("co"),
                                  lse=o.get("cl"), ws=ws[spec.DENSE_WINDOW])
        o["p"] = spec.prefix_decode_attn(q, Kp, Vp, s["K"], s["V"], lens, out=o.get("po"),
                                         lse=o.get("pl"), ws=ws[spec.DENSE_PREFIX_DECODE])

    eager = {k: v.clone() for k, v in state.items()}
    fixed = {nm + "o": torch.zeros_like(q, dtype=torch.float32) for nm in "awp"}
    fixed.update({nm + "l": torch.zeros(q.shape[:-1], device=dev) for nm in "awp"})
    fixed.update(co=torch.zeros_like(qc), cl=torch.zeros(qc.shape[:-1], device=dev))
    warm = {k: v.clone() for k, v in state.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm, dict(fixed))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs.update(fixed)
        step(state, outs)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in list(state.items()) + list(fixed.items())}
        want = {}
        step(eager, want)
        torch.cuda.synchronize()
        for k in state:
            assert same_bits(got[k], eager[k]), (i, k)
        for nm in "awcp":
            assert torch.equal(got[nm + "o"], want[nm][0]), (i, nm)
            assert torch.equal(got[nm + "l"], want[nm][1]), (i, nm)


def test_other_stream_and_two_at_once(dev):
    """Calls on two streams at once, each with its own workspace and outputs."""
    n, B, H_q, H_kv, cap = 1, 4, 32, 8, 2000
    K, V = cache(n, B, cap, H_kv, 171, dev)
    Kp, Vp = (normal((n, 1500, H_kv, D), 173 + i, dev) for i in range(2))
    q = normal((n, B, H_q, D), 175, dev)
    qc = normal((n, B, 40, H_q, D), 176, dev)
    lens = i32([2000, 1500, 3, 0], dev)
    torch.cuda.synchronize()
    calls = [lambda: spec.window_attn(qc, K, V, lens, 700, n_sink=4),
             lambda: spec.prefix_decode_attn(q, Kp, Vp, K, V, lens),
             lambda: spec.window_decode_attn(q, K, V, lens, 700, n_sink=4),
             lambda: spec.accum_decode_attn(q, K, V, lens, torch.zeros((n, B, 1, cap), device=dev))]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for c, s in zip(calls, streams):
        with torch.cuda.stream(s):
            got.append(c())
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_native_marshalling_equals_ctypes(dev, monkeypatch):
    """Calls that hand over every buffer, with and without the native marshalling."""
    n, B, H_q, H_kv, cap, T, P = 2, 3, 16, 4, 200, 7, 90
    K, V = cache(n, B, cap, H_kv, 181, dev)
    Kp, Vp = (normal((n, P, H_kv, D), 183 + i, dev) for i in range(2))
    q, qc = normal((n, B, H_q, D), 185, dev), normal((n, B, T, H_q, D), 186, dev)
    kv = normal((2, n, B, 3, H_kv, D), 187, dev)
    lens, rows, keep = i32([200, 77, 0], dev), i32([7, 3, 0], dev), i32([200, 70, 9], dev)

    def all_calls():
        w = torch.ones((n, B, H_kv, cap), device=dev)
        o = [torch.zeros(q.shape, device=dev) for _ in range(3)]
        z = [torch.zeros(q.shape[:-1], device=dev) for _ in range(3)]
        oc, zc = torch.zeros_like(qc), torch.zeros(qc.shape[:-1], device=dev)
        ws = torch.empty(1 << 24, dtype=torch.uint8, device=dev)
        spec.window_decode_attn(q, K, V, lens, 50, n_sink=3, scale=0.1, out=o[0], lse=z[0], ws=ws)
        spec.window_attn(qc, K, V, lens, 50, n_sink=3, q_lens=rows, scale=0.1, out=oc, lse=zc,
                         ws=ws)
        spec.prefix_decode_attn(q, Kp, Vp, K, V, lens, prefix_len=i32([80], dev), scale=0.1,
                                out=o[1], lse=z[1], ws=ws)
        spec.accum_decode_attn(q, K, V, lens, w, scale=0.1, out=o[2], lse=z[2], ws=ws)
        Ke, Ve, t, c = K.clone(), V.clone(), w.int(), lens.clone()
        spec.evict(Ke, Ve, w, t, c, keep, i32([300, 77, 0], dev), k_new=kv[0], v_new=kv[1],
                   n_new=i32([3, 1, 2], dev), n_recent=5, n_sink=2, ws=ws)
        return o + z + [oc, zc, w, Ke, Ve, t, c]

    assert spec._fast is not None
    taken = []
    for name in ("window_decode", "window", "prefix_decode", "accum_decode", "evict"):
        f = getattr(spec._fast, name)
        monkeypatch.setattr(spec._fast, name,
                            lambda *a, f=f, name=name: taken.append((name, r := f(*a))) or r)
    native = all_calls()
    assert taken == [(nm, 0) for nm in ("window_decode", "window", "prefix_decode", "accum_decode",
                                        "evict")]
    monkeypatch.setattr(spec, "_fast", None)
    for a, b in zip(native, all_calls()):
        assert same_bits(a, b)


def test_refusals_name_the_argument(dev):
    K, V = cache(1, 2, 40, 4, 191, dev)
    q, lens = normal((1, 2, 8, D), 192, dev), i32([40, 3], dev)
    w = torch.zeros((1, 2, 4, 40), device=dev)
    ws = torch.empty(8, dtype=torch.uint8, device=dev)
    for bad, call in (
            ("q must", lambda: spec.window_decode_attn(q[:, :1], K, V, lens, 8)),
            ("seq_lens", lambda: spec.window_decode_attn(q, K, V, lens[:1], 8)),
            ("out", lambda: spec.window_decode_attn(q, K, V, lens, 8, out=q)),
            ("same shape", lambda: spec.window_decode_attn(q, K, V[:, :, :30], lens, 8)),
            ("INVALID", lambda: spec.window_decode_attn(q, K, V, lens, 0)),
            ("UNSUPPORTED", lambda: spec.window_decode_attn(
                q[..., :64].contiguous(), K[..., :64].contiguous(), V[..., :64].contiguous(), lens,
                8)),
            ("K_prefix", lambda: spec.prefix_decode_attn(q, K[0], V[0], K, V, lens)),
            ("weights", lambda: spec.accum_decode_attn(q, K, V, lens, w[:, :, :2])),
            ("workspace", lambda: spec.accum_decode_attn(q, K, V, lens, w, ws=ws)),
            ("tokens", lambda: spec.evict(K, V, w, w.int()[:, :1], lens, lens, lens)),
            ("together", lambda: spec.evict(K, V, w, w.int(), lens, lens, lens, k_new=K)),
            ("INVALID", lambda: spec.evict(K, V, w, w.int(), lens, lens, lens, n_recent=-1))):
        with pytest.raises((ValueError, TypeError, spec.SpecError), match=bad):
            call()
