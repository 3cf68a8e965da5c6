"""The entry points over caches that are read in full within bounds that come from each
query's own logits (dense_bounds): inputs whose largest logit rises again and again along
the tokens, by more than a running maximum may lag, and weights whose low bits are known."""
import math

import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from tests import dense_bounds as db
from tests.dense_bounds import D
from tests.gpu_helpers import announce, f64, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def normal(shape, seed, dev, sd=1.0):
    g = torch.Generator().manual_seed(seed)
    return (sd * torch.randn(shape, generator=g)).to(torch.bfloat16).to(dev)


def rising(n, B, L, H_kv, seed, dev, total):
    """K, V: log2-unit logits of queries() rise by 10 every 64 tokens, for three such blocks,
    and by 9 every sixth of `total` tokens; normal values beside that."""
    K, V = normal((n, B, L, H_kv, D), seed, dev, 0.5), normal((n, B, L, H_kv, D), seed + 1, dev)
    t = torch.arange(L, device=dev)
    level = 10.0 * (t // 64 % 3) + 9.0 * (6 * t // max(total, 1))
    # 16 y / sqrt(128) log2(e) = level
    K[..., 0] = (level / (16 * db.SCALE * math.log2(math.e))).to(torch.bfloat16)[None, None, :,
                                                                                None]
    return K, V


def queries(shape, seed, dev):
    q = normal(shape, seed, dev)
    q[..., 0] = 16.0
    return q


def compare(what, out, lse, q, k, v, parts, rounded=False):
    """out, lse [H][D], [H] of queries q [H][D] over rows k, v."""
    for h in range(q.shape[0]):
        want, wlse, tol, tol_lse = db.attend(q[h], k, v, parts)
        if rounded:
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
        err = np.abs(out[h] - want)
        assert (err <= tol).all(), (what, h, float((err / tol).max()))
        assert abs(lse[h] - wlse) <= tol_lse, (what, h, abs(lse[h] - wlse) / tol_lse)


def seen(p, window, n_sink):
    t = np.arange(p + 1)
    return t[(t < n_sink) | (t > p - window)]


# ------------------------------------------------------------------ rising logits

DECODE = [
    # layers, H_q, H_kv, cap, lens, window, sinks
    (1, 32, 8, 900, [900, 333, 1, 64], 700, 4),                        # one group
    (1, 8, 2, 20011, [20011, 15000], 20011, 0),                        # in parts
    (4, 6, 2, 700, [700 - b for b in range(64)], 600, 3),              # two groups
    (32, 32, 8, 1200, [1200 - 50 * b for b in range(8)], 1000, 4),     # four
    (8, 16, 4, 2100, [2100 - 97 * b for b in range(16)], 1000, 4),     # ... in parts
    (1, 24, 1, 3000, [3000, 2999], 3000, 0),                           # 24 heads a KV head
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_l{c[3]}_w{c[5]}")
def test_decode(dev, case):
    n, H_q, H_kv, cap, lens, window, sinks = case
    announce(f"rising decode {case}")
    B, G = len(lens), H_q // H_kv
    K, V = rising(n, B, cap, H_kv, 41, dev, cap)
    q = queries((n, B, H_q, D), 43, dev)
    win = spec.window_decode_attn(q, K, V, i32(lens, dev), window, n_sink=sinks)
    w = torch.zeros((n, B, 1, cap), device=dev)
    acc = spec.accum_decode_attn(q, K, V, i32(lens, dev), w)
    for layer, b, g in ((0, 0, 0), (n - 1, B - 1, H_kv - 1), (n // 2, B // 2, H_kv // 2)):
        heads = slice(g * G, (g + 1) * G)
        for what, (out, lse), rows in (("window", win, seen(lens[b] - 1, window, sinks)),
                                       ("accum", acc, np.arange(lens[b]))):
            compare((what, layer, b, g), f64(out[layer, b, heads]), f64(lse[layer, b, heads]),
                    f64(q[layer, b, heads]), f64(K[layer, b, :, g])[rows],
                    f64(V[layer, b, :, g])[rows], 3)


WINDOW = [
    # H_q, H_kv, cap, T, lens, window, sinks
    (8, 8, 700, 40, [700, 650], 700, 0),              # 32 rows, in parts
    (3, 1, 400, 100, [400, 399], 77, 5),              # 32 rows
    (28, 4, 1500, 257, [1500, 257], 777, 3),          # 64 rows
    (6, 2, 9021, 126, [9020], 4537, 5),               # ... in parts
    (32, 8, 2048, 2048, [2001], 2048, 0),             # 128 rows
    (64, 8, 11287, 77, [11287, 9000, 77], 7663, 4),   # ... in parts
    (24, 8, 3751, 740, [3751, 3000, 741], 3273, 4),   # 256 rows
    (32, 8, 8192, 512, [8192], 8192, 0),              # ... in parts
]


@pytest.mark.parametrize("case", WINDOW, ids=lambda c: f"h{c[0]}_{c[1]}_l{c[2]}_t{c[3]}_w{c[5]}")
def test_window(dev, case):
    H_q, H_kv, cap, T, lens, window, sinks = case
    announce(f"rising window {case}")
    B, G = len(lens), H_q // H_kv
    K, V = rising(1, B, cap, H_kv, 51, dev, cap)
    q = queries((1, B, T, H_q, D), 53, dev)
    out, lse = spec.window_attn(q, K, V, i32(lens, dev), window, n_sink=sinks)
    for b, g in {(0, 0), (B - 1, H_kv - 1)}:
        heads = slice(g * G, (g + 1) * G)
        k, v = f64(K[0, b, :, g]), f64(V[0, b, :, g])
        for i in sorted({0, 1, T // 3, T // 2, T - 2, T - 1}):
            rows = seen(lens[b] - T + i, window, sinks)
            if len(rows):
                compare((b, g, i), f64(out[0, b, i, heads]), f64(lse[0, b, i, heads]),
                        f64(q[0, b, i, heads]), k[rows], v[rows], 1, rounded=True)


PREFIX = [
    # H_q, H_kv, P, cap, lens: 32, 64, 128, 256 rows and two row tiles, own tokens in one
    # column group and in four
    (32, 8, 20011, 777, [777, 400, 0, 5]),
    (32, 8, 4097, 300, [300, 17] * 8),
    (64, 16, 2000, 700, [700, 5, 0, 699] * 5),
    (32, 8, 9000, 300, [300, 0, 17, 299] * 16),
    (128, 1, 3000, 64, [64] * 5),
]


@pytest.mark.parametrize("case", PREFIX, ids=lambda c: f"h{c[0]}_{c[1]}_p{c[2]}_b{len(c[4])}")
@pytest.mark.parametrize("upper", ["prefix", "own"])
def test_prefix(dev, case, upper):
    """The largest logits in the prefix, or (its keys negated) in the sequences' own tokens."""
    H_q, H_kv, P, cap, lens = case
    announce(f"rising prefix {case} {upper}")
    B, G = len(lens), H_q // H_kv
    K, V = rising(1, B, cap, H_kv, 61, dev, cap)
    Kp, Vp = (t[:, 0] for t in rising(1, 1, P, H_kv, 63, dev, P))
    (Kp if upper == "own" else K)[..., 0] *= -1.0
    q = queries((1, B, H_q, D), 65, dev)
    out, lse = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32(lens, dev))
    for b, g in {(0, 0), (B - 1, H_kv - 1), (B // 2, H_kv // 2)}:
        heads = slice(g * G, (g + 1) * G)
        compare((b, g), f64(out[0, b, heads]), f64(lse[0, b, heads]), f64(q[0, b, heads]),
                np.concatenate([f64(Kp[0, :, g]), f64(K[0, b, :lens[b], g])]),
                np.concatenate([f64(Vp[0, :, g]), f64(V[0, b, :lens[b], g])]),
                3 if B * G <= 32 else 2)


# ------------------------------------------------------------------ normal values

def test_long_caches(dev):
    """Normal values on the lengths whose tails a wider tolerance would hide."""
    announce("long caches")
    H_q, H_kv, P, B = 32, 8, 20011, 15
    Kp, Vp = (normal((1, P, H_kv, D), 71 + i, dev) for i in range(2))
    K, V = (normal((1, B, 777, H_kv, D), 73 + i, dev) for i in range(2))
    q = normal((1, B, H_q, D), 75, dev)
    lens = [777, 5, 400] * 5
    out, lse = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32(lens, dev))
    few = spec.prefix_decode_attn(q[:, :4].contiguous(), Kp, Vp, K[:, :4], V[:, :4],
                                  i32(lens[:4], dev))
    one = spec.window_decode_attn(q[:, :1].contiguous(), Kp[:, None], Vp[:, None], i32([P], dev), P)
    for g in range(0, H_kv, 3):
        heads = slice(4 * g, 4 * g + 4)
        kp, vp = f64(Kp[0, :, g]), f64(Vp[0, :, g])
        compare("window", f64(one[0][0, 0, heads]), f64(one[1][0, 0, heads]), f64(q[0, 0, heads]),
                kp, vp, 3)
        for b in (0, 3, 14):
            k = np.concatenate([kp, f64(K[0, b, :lens[b], g])])
            v = np.concatenate([vp, f64(V[0, b, :lens[b], g])])
            compare(("prefix", b), f64(out[0, b, heads]), f64(lse[0, b, heads]),
                    f64(q[0, b, heads]), k, v, 2)
            if b < 4:
                compare(("few", b), f64(few[0][0, b, heads]), f64(few[1][0, b, heads]),
                        f64(q[0, b, heads]), k, v, 3)


# ------------------------------------------------------------------ the weights' low bits

def ratios(out, w, parts, tokens):
    """out [..][H][D], w [H]."""
    got = out[..., 64:] / out[..., :64]
    err = np.abs(got / w[:, None] - 1)
    assert (err <= db.two_level_tolerance(tokens, parts)).all(), float(err.max() / db.U)


@pytest.mark.parametrize("n,B,H_q,H_kv,L", [(1, 2, 8, 2, 256), (1, 1, 8, 8, 512),
                                            (4, 64, 6, 2, 512), (32, 8, 32, 8, 256),
                                            (2, 2, 24, 1, 512)])
def test_decode_weights_in_three_numbers(dev, n, B, H_q, H_kv, L):
    """One, two and four column groups beside each other; the logits of the accumulated
    weights in memory and in LDS."""
    announce(f"low bits decode {n} {B} {H_q} {H_kv} {L}")
    x, w = db.two_level_queries(H_q)
    K, V = db.two_level_cache(n, B, L, H_kv, dev)
    q = torch.zeros((n, B, H_q, D), dtype=torch.bfloat16, device=dev)
    q[..., 0] = torch.from_numpy(x).to(dev, torch.bfloat16)
    lens = i32([L] * B, dev)
    sums = torch.zeros((n, B, H_kv, L), device=dev)
    out, _ = spec.window_decode_attn(q, K, V, lens, L)
    ratios(f64(out), w, 3, L // 128)
    out, _ = spec.accum_decode_attn(q, K, V, lens, sums)
    ratios(f64(out), w, 3, L // 128)
    # the accumulated weights themselves: w / (L / 2 (1 + w)) a head, within the roundings of
    # the argument, two exponentials and a logarithm (dense_bounds) and those of the sums
    G = H_q // H_kv
    want = w / (L / 2 * (1 + w)), 1 / (L / 2 * (1 + w))
    for t, p in ((1, want[0]), (0, want[1])):
        p = p.reshape(H_kv, G).sum(1)
        err = np.abs(f64(sums[:, :, :, t::2]) - p[:, None])
        assert (err <= (5 * math.log2(L) + 16 + G + math.sqrt(L)) * db.U * p[:, None]).all()


@pytest.mark.parametrize("B,G,parts", [(2, 4, 3), (8, 4, 3), (16, 4, 2), (32, 4, 2), (64, 4, 2),
                                       (3, 128, 2)])
def test_prefix_weights_in_three_numbers_and_two(dev, B, G, parts):
    """Three for up to 32 rows on the prefix, two above that."""
    announce(f"low bits prefix {B} {G}")
    H_kv = 2
    x, w = db.two_level_queries(G * H_kv)
    K, V = db.two_level_cache(1, B, 256, H_kv, dev)
    Kp, Vp = (t[:, 0] for t in db.two_level_cache(1, 1, 256, H_kv, dev))
    q = torch.zeros((1, B, G * H_kv, D), dtype=torch.bfloat16, device=dev)
    q[..., 0] = torch.from_numpy(x).to(dev, torch.bfloat16)
    out, _ = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32([256] * B, dev))
    ratios(f64(out), w, parts, 4)
