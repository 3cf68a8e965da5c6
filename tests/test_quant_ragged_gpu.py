"""Decode attention over caches in 4 and 8 bits of ragged lengths, whose parts a launch deals
to the sequences by their lengths: no token is missed or counted twice, however the
lengths lie.

Counted tokens (dense_bounds): keys of zeros, so that every visible token weighs 1, and rows
of V with one value each.  The values 1 to 1.75 and 0 are elements of 8 bits; in 4 bits (whose
elements are 1, 1.5 ..) a token has 1 in its dimension.  A sum of n such values is exact in
fp32, n and its reciprocal take a rounding each and their product another: an output is off
by 4 U of itself, the log-sum-exp log(n) by 6 U, as dense_bounds works out."""
import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from tests import dense_bounds as db
from tests.gpu_helpers import announce, f64, need_gpu
from tests.quant_helpers import D, compare, i32, normal, read_head

pytestmark = pytest.mark.gpu

# layers, sequences, tokens, KV heads: all dealt
SHAPES = [(1, 64, 8000, 1), (2, 64, 4000, 2), (2, 5, 16000, 8), (4, 2, 16000, 8), (8, 3, 8192, 8),
          (4, 5, 40000, 1)]


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


def lengths(kind, B, L, rng):
    if kind == "equal":
        return [L] * B
    if kind == "none":
        return [0] * B
    if kind == "one":
        return [0] * (B - 1) + [L]
    if kind == "few":                # fewer chunks than parts
        return [1 + b % 3 for b in range(B)]
    if kind == "linear":
        return [L * (b + 1) // B for b in range(B)]
    if kind == "two":
        return [L if b % 3 == 0 else 33 for b in range(B)]
    return rng.integers(0, L + 1, B).tolist()


@pytest.mark.parametrize("bits", (4, 8))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n{}_b{}_l{}_h{}".format(*s))
def test_every_token_counts_once(dev, shape, bits):
    n, B, L, H_kv = shape
    G = 2
    t = torch.arange(L, device=dev)
    a = db.amplitude(t) if bits == 8 else torch.ones(L, device=dev)
    K = torch.zeros((1, 1, L, H_kv, D), dtype=torch.bfloat16, device=dev)
    V = torch.zeros_like(K)
    for g in range(H_kv):
        V[0, 0, t, g, (t + 37 * g) % D] = a.to(torch.bfloat16)
    one = spec.QuantCache(1, 1, L, H_kv, bits=bits, device=dev)
    spec.quant_append(one, K, V, i32([0], dev))
    assert torch.equal(spec.quant_read(one, i32([L], dev))[1], V)
    cache = spec.QuantCache.of(*(x.expand(n, B, *x.shape[2:]).contiguous()
                                 for x in (one.k, one.v, one.scales)))
    table = torch.zeros((L + 1, D), dtype=torch.float64, device=dev)
    table[t + 1, t % D] = a.double()
    table = table.cumsum(0)
    q = normal((n, B, G * H_kv, D), 401, dev)
    rng = np.random.default_rng(402)
    idx = i32(np.broadcast_to(np.arange(L), (B, L)).copy(), dev)
    for kind in ("equal", "none", "one", "few", "linear", "two", "random"):
        announce(f"deal {shape} {bits} {kind}")
        lens = lengths(kind, B, L, rng)
        ln = i32(lens, dev)
        m = ln.long()
        for window, sinks in ((None, 0), (L - 1, 40), ("selected", 0)):
            if window == "selected":
                out, lse = spec.quant_sparse_decode_attn(q, cache, ln, idx)
            else:
                out, lse = spec.quant_decode_attn(q, cache, ln, window=window, n_sink=sinks)
            want = table[m] / m.clamp(min=1)[:, None]
            want_lse = db.lse_of(m)
            for g in range(H_kv):
                hs = slice(g * G, (g + 1) * G)
                w = want.roll(37 * g, 1)[None, :, None]
                err = (out[:, :, hs].double() - w).abs()
                assert (err <= 4 * db.U * w).all(), (kind, window, g)
                z = lse[:, :, hs].double()
                zw = want_lse[None, :, None].expand_as(z)
                same = (z == zw)
                assert (same | ((z - zw).abs() <= 6 * db.U * zw.abs())).all(), (kind, window, g)


@pytest.mark.parametrize("bits", (4, 8))
def test_a_window_of_ragged_lengths(dev, bits):
    """Sinks and a window in long caches of lengths around both."""
    announce(f"ragged window {bits}")
    n, B, L, H_kv, G, window, sinks = 8, 6, 12000, 8, 4, 6000, 70
    t = torch.arange(L, device=dev)
    K = torch.zeros((1, 1, L, H_kv, D), dtype=torch.bfloat16, device=dev)
    V = torch.zeros_like(K)
    V[0, 0, t, :, t % D] = 1.0
    one = spec.QuantCache(1, 1, L, H_kv, bits=bits, device=dev)
    spec.quant_append(one, K, V, i32([0], dev))
    cache = spec.QuantCache.of(*(x.expand(n, B, *x.shape[2:]).contiguous()
                                 for x in (one.k, one.v, one.scales)))
    table = torch.zeros((L + 1, D), dtype=torch.float64, device=dev)
    table[t + 1, t % D] = 1.0
    table = table.cumsum(0)
    lens = [12000, 6071, 6070, 69, 0, 9001]
    q = normal((n, B, G * H_kv, D), 403, dev)
    out, lse = spec.quant_decode_attn(q, cache, i32(lens, dev), window=window, n_sink=sinks)
    want, m = db.counted_window(table, torch.tensor(lens, device=dev) - 1, window, sinks)
    w = want[None, :, None]
    assert ((out.double() - w).abs() <= 4 * db.U * w).all()
    zw = db.lse_of(m)[None, :, None].expand_as(lse)
    assert ((lse == zw) | ((lse.double() - zw).abs() <= 6 * db.U * zw.abs())).all()


def test_other_lengths_beside(dev):
    """The same lengths give the same bits; other lengths of the other sequences may divide a
    sequence differently, and its result stays within its bounds."""
    announce("ragged, other lengths beside")
    n, B, L, H_kv, G = 2, 5, 16000, 8, 4
    g = torch.Generator().manual_seed(404)
    k, v = (torch.randint(0, 256, (n, B, L, H_kv, 64), generator=g, dtype=torch.uint8).to(dev)
            for _ in range(2))
    s = torch.randint(123, 127, (n, B, L, H_kv, 2, 4), generator=g, dtype=torch.uint8).to(dev)
    cache = spec.QuantCache.of(k, v, s)
    q = normal((n, B, G * H_kv, D), 405, dev)
    K, V = read_head(cache, 1, 0, 3)
    for others in ([9000, 30, 12345, 700], [1, 16000, 0, 5], [0, 0, 0, 0]):
        lens = i32([16000] + others, dev)
        out, lse = spec.quant_decode_attn(q, cache, lens)
        again = spec.quant_decode_attn(q, cache, lens)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
        hs = slice(3 * G, 4 * G)
        compare(others, f64(out[1, 0, hs]), f64(lse[1, 0, hs]), f64(q[1, 0, hs]), K, V)
