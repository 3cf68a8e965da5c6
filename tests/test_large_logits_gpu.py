"""Logits of 2^20 to 2^100 in both signs, finite and far from any other: what is attended is
known exactly.

Queries have one dimension that is not 0, so that a logit is one product, exact in fp32 for
bf16 operands of these sizes, and tokens have the same logit or ones that differ by one part
in 2^8 at least, 2^8 log2 units or more, so that every weight is that of the greatest or 0.
An output is then the mean of the m rows of V whose logit is the greatest: sums of m
terms (m - 1 roundings, each U of a partial sum, which the sum of absolute values bounds), the
reciprocal of m, and its product with the sum: (m + 2) U of the mean absolute value.  Rows
that join in any order take no more.  The log-sum-exp is scale times that logit plus log(m):
the scale, log2(e), their product, that with the logit, the sum with log2(m), ln(2) and the
product with it are a rounding each, 7 U of it, and log2(m) is off by less than 2^-18: 8 U are
allowed and 2^-18 more.  Where the greatest logits are 0, they are the same with a
log-sum-exp of log(m).  Weights that enter the products rounded to bf16 are off by 2^-8 of
themselves, as two bf16 numbers by 2^-17, and an output in bf16 by 2^-8 of itself."""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from tests import dense_bounds as db
from tests.gpu_helpers import announce, f64, need_gpu
from tests.quant_helpers import D, i32, normal, read

pytestmark = pytest.mark.gpu

EXPONENTS = (20, 23, 24, 27, 30, 31, 32, 33, 34, 36, 40, 52, 64, 100)


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


def queries(shape, e, dev):
    """Of dimension 0 alone: 2^(e + 2) to 2^(e + 3), both signs in turn."""
    q = torch.zeros(shape, dtype=torch.float64)
    h = torch.arange(shape[-2])
    q[..., 0] = (1 - 2 * (h % 2)) * 2.0 ** (e + 2) * (1 + 23 * h % 128 / 128.0)
    q = q.to(torch.bfloat16)
    return q.to(dev)


def keys(kind, shape, seed, dev):
    """Normal rows, but for dimension 0: levels 1 to 2 of every token; levels of some, beside
    0 of the others; or levels of the first tokens only."""
    n, B, L, H_kv = shape
    K = normal((*shape, D), seed, dev)
    rng = np.random.default_rng(seed)
    x = 1 + rng.integers(0, 128, shape) / 128.0
    if kind == "some":
        x[rng.random(shape) < 0.7] = 0
    if kind == "first":
        x[:, :, L // 2:] = 0
    K[..., 0] = torch.tensor(x).to(torch.bfloat16).to(dev)
    return K


def check(what, out, lse, q, k, v, skip=(), more=0.0):
    """out [D], lse of one query q [D] over rows k, v [n][D] (float64); dimensions `skip` of
    the output are not looked at; more: what weights and output are off by beside fp32."""
    if len(k) == 0:
        assert (out == 0).all() and lse == -math.inf, what
        return
    s = db.SCALE * (k[:, 0] * q[0])
    top = s.max()
    near = s == top
    rest = s[~near]
    assert len(rest) == 0 or rest.max() < top - 1000, what   # the inputs are as described
    dims = [d for d in range(D) if d not in skip]
    rows = v[near]
    m = len(rows)
    err = np.abs(out - rows.mean(0))[dims]
    tol = ((m + 2) * db.U + more) * np.abs(rows).mean(0)[dims]
    assert (err <= tol).all(), (what, m, top, out[dims][:4], rows.mean(0)[dims][:4])
    want = top + math.log(m)
    assert abs(lse - want) <= 8 * db.U * abs(want) + 2.0 ** -18, (what, m, lse, want)


# ------------------------------------------------------------------ caches in 4 and 8 bits

# layers, KV heads, query heads of each, tokens, lengths
QUANT = [(1, 2, 4, 40, [40, 1, 33]), (1, 3, 2, 200, [200, 65, 0]), (2, 2, 8, 300, [300, 17]),
         (1, 8, 16, 700, [700]), (1, 4, 1, 4000, [4000, 900, 2]), (1, 2, 20, 150, [150, 150])]


@pytest.mark.parametrize("bits", (4, 8))
@pytest.mark.parametrize("e", EXPONENTS)
def test_quantised_caches(dev, e, bits):
    for case, (n, H_kv, G, L, lens) in enumerate(QUANT):
        B = len(lens)
        q = queries((n, B, G * H_kv, D), e, dev)
        for j, kind in enumerate(("all", "some", "first")):
            announce(f"large logits {bits} 2^{e} {QUANT[case]} {kind}")
            K = keys(kind, (n, B, L, H_kv), 500 + 10 * case + j, dev)
            V = normal((n, B, L, H_kv, D), 600 + 10 * case + j, dev)
            cache = spec.QuantCache(n, B, L, H_kv, bits=bits, device=dev)
            spec.quant_append(cache, K, V, i32([0] * B, dev))
            rng = np.random.default_rng(700 + case)
            idx = np.full((B, L), -1)
            for b, m in enumerate(lens):
                idx[b, :m] = np.sort(rng.choice(L, m, replace=False))
            dense = [f64(t) for t in spec.quant_decode_attn(q, cache, i32(lens, dev))]
            sparse = [f64(t) for t in spec.quant_sparse_decode_attn(q, cache, i32(lens, dev),
                                                                    i32(idx, dev))]
            Kh, Vh = read(cache)
            qh = f64(q)
            for layer in range(n):
                for b, m in enumerate(lens):
                    for h in range(G * H_kv):
                        g = h // G
                        for what, (out, lse), rows in (("dense", dense, np.arange(m)),
                                                       ("sparse", sparse, idx[b, :m])):
                            check((what, QUANT[case], kind, layer, b, h), out[layer, b, h],
                                  lse[layer, b, h], qh[layer, b, h], Kh[layer, b, rows, g],
                                  Vh[layer, b, rows, g])


@pytest.mark.parametrize("bits", (4, 8))
@pytest.mark.parametrize("e", EXPONENTS)
def test_quantised_caches_beside_a_nan(dev, e, bits):
    """A group of V that is NaN sends the sums the way of the rare ones: the other groups'
    outputs are as before."""
    announce(f"large logits {bits} 2^{e} beside a NaN")
    n, B, L, H_kv, G = 1, 2, 100, 2, 4
    lens = [100, 61]
    q = queries((n, B, G * H_kv, D), e, dev)
    K, V = keys("some", (n, B, L, H_kv), 511, dev), normal((n, B, L, H_kv, D), 611, dev)
    V[:, :, 5, :, 40] = math.nan          # dimensions 32 to 63
    cache = spec.QuantCache(n, B, L, H_kv, bits=bits, device=dev)
    spec.quant_append(cache, K, V, i32([0] * B, dev))
    out, lse = (f64(t) for t in spec.quant_decode_attn(q, cache, i32(lens, dev)))
    Kh, Vh = read(cache)
    for b, m in enumerate(lens):
        for h in range(G * H_kv):
            check((b, h), out[0, b, h], lse[0, b, h], f64(q[0, b, h]), Kh[0, b, :m, h // G],
                  Vh[0, b, :m, h // G], skip=range(32, 64))


# ------------------------------------------------------------------ caches in bf16

# layers, KV heads, query heads of each, tokens, lengths
BF16 = [(1, 2, 4, 40, [40, 1, 33]), (2, 3, 8, 300, [300, 65, 0]), (1, 1, 16, 1500, [1500, 999])]


def bf16_case(case, j, kind, odd, dev):
    """K, V; odd: an infinity in dimension 40 of V, which sends the sums the way of the rare
    ones."""
    n, H_kv, _, L, lens = BF16[case]
    K = keys(kind, (n, len(lens), L, H_kv), 520 + 10 * case + j, dev)
    V = normal((n, len(lens), L, H_kv, D), 620 + 10 * case + j, dev)
    if odd:
        V[:, :, 0, :, 40] = math.inf
    Vh = f64(V)
    return K, V, f64(K), np.where(np.isfinite(Vh), Vh, 0)


@pytest.mark.parametrize("odd", (False, True), ids=("finite", "inf"))
@pytest.mark.parametrize("e", EXPONENTS)
def test_a_decode_step(dev, e, odd):
    """Over all rows, and over selected ones."""
    skip = (40,) if odd else ()
    for case, (n, H_kv, G, L, lens) in enumerate(BF16):
        q = queries((n, len(lens), G * H_kv, D), e, dev)
        for j, kind in enumerate(("all", "some", "first")):
            announce(f"large logits bf16 2^{e} {BF16[case]} {kind} {skip}")
            K, V, Kh, Vh = bf16_case(case, j, kind, odd, dev)
            rng = np.random.default_rng(720 + case)
            idx = np.full((len(lens), L), 0)
            for b, m in enumerate(lens):
                idx[b, :m] = np.sort(rng.choice(L, m, replace=False))
            dense = [f64(t) for t in spec.window_decode_attn(q, K, V, i32(lens, dev), window=L)]
            sparse = [f64(t) for t in spec.sparse_decode_attn(q, K, V, i32(lens, dev),
                                                              idx=i32(idx, dev))]
            qh = f64(q)
            for layer, b, h in itertools.product(range(n), range(len(lens)), range(G * H_kv)):
                for what, (out, lse), rows, more in (
                        ("dense", dense, np.arange(lens[b]), 0.0),
                        ("sparse", sparse, idx[b, :lens[b]], 2.0 ** -17)):
                    check((what, BF16[case], kind, layer, b, h), out[layer, b, h],
                          lse[layer, b, h], qh[layer, b, h], Kh[layer, b, rows, h // G],
                          Vh[layer, b, rows, h // G], skip, more)


@pytest.mark.parametrize("odd", (False, True), ids=("finite", "inf"))
@pytest.mark.parametrize("e", EXPONENTS)
def test_a_chunk_of_queries(dev, e, odd):
    skip, T = (40,) if odd else (), 5
    for case, (n, H_kv, G, L, lens) in enumerate(BF16):
        q = queries((n, len(lens), T, G * H_kv, D), e, dev)
        for j, kind in enumerate(("all", "some", "first")):
            announce(f"large logits chunk 2^{e} {BF16[case]} {kind} {skip}")
            K, V, Kh, Vh = bf16_case(case, j, kind, odd, dev)
            own = [min(T, m) for m in lens]
            out, lse = (f64(t) for t in spec.window_attn(q, K, V, i32(lens, dev), window=L,
                                                         q_lens=i32(own, dev)))
            qh = f64(q)
            for layer, b, h in itertools.product(range(n), range(len(lens)), range(G * H_kv)):
                for i in range(own[b]):
                    p = lens[b] - own[b] + i + 1
                    check((BF16[case], kind, layer, b, i, h), out[layer, b, i, h],
                          lse[layer, b, i, h], qh[layer, b, i, h], Kh[layer, b, :p, h // G],
                          Vh[layer, b, :p, h // G], skip, 2.0 ** -7)   # weights and output


@pytest.mark.parametrize("odd", (False, True), ids=("finite", "inf"))
@pytest.mark.parametrize("e", EXPONENTS)
def test_a_shared_prefix(dev, e, odd):
    """Levels of the prefix from 1, of the own tokens from 2: the greatest logits are
    those of the one or the other."""
    skip = (40,) if odd else ()
    for n, H_kv, G, P, L, lens in ((1, 2, 4, 700, 90, [90, 0, 33]), (2, 1, 16, 100, 50, [50] * 6)):
        announce(f"large logits prefix 2^{e} {P} {L} {skip}")
        B = len(lens)
        q = queries((n, B, G * H_kv, D), e, dev)
        Kp, Vp = keys("all", (n, 1, P, H_kv), 541, dev)[:, 0], normal((n, P, H_kv, D), 641, dev)
        K, V = keys("all", (n, B, L, H_kv), 542, dev), normal((n, B, L, H_kv, D), 642, dev)
        K[..., 0] *= 2
        if odd:
            Vp[:, 3, :, 40] = math.inf
            V[:, :, 2, :, 40] = -math.inf
        out, lse = (f64(t) for t in spec.prefix_decode_attn(q, Kp.contiguous(), Vp, K, V,
                                                            i32(lens, dev)))
        ph, qh, oh = (f64(Kp), f64(Vp)), f64(q), (f64(K), f64(V))
        for layer in range(n):
            for b, m in enumerate(lens):
                for h in range(G * H_kv):
                    g = h // G
                    k, v = (np.concatenate([x[layer, :, g], y[layer, b, :m, g]])
                            for x, y in zip(ph, oh))
                    check((P, layer, b, h), out[layer, b, h], lse[layer, b, h], qh[layer, b, h],
                          k, v, skip, 2.0 ** -17)
