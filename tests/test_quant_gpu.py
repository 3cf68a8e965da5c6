"""Caches held in 4 or 8 bits: quantised as they are written, read back, attended.

What is written and read back is compared bit for bit with the oracle's.  Attention is
within the bounds that dense_bounds.attend derives from each query's own logits, over the
oracle's values of the held rows: K and V enter exactly, the weights as three bf16
numbers."""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from oracle import quant_oracle as qo
from tests.gpu_helpers import announce, f64, need_gpu
from tests.quant_helpers import D, compare, held, i32, normal, read, seen

pytestmark = pytest.mark.gpu

BITS = (4, 8)


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


def bits_of(t):
    return t.contiguous().view(torch.int16)


# ------------------------------------------------------------------ written

def written(x, bits, dev):
    """Rows x [rows][D] bf16 through a cache of one sequence and head: codes, scales, read."""
    rows = x.shape[0]
    cache = spec.QuantCache(1, 1, rows, 1, bits=bits, device=dev)
    new = x.to(dev)[None, None, :, None]
    spec.quant_append(cache, new, new.flip(2).contiguous(), i32([0], dev))
    K, V = spec.quant_read(cache, i32([rows], dev))
    for t, j in ((cache.k, 0), (cache.v, 1)):
        y = f64(x if j == 0 else x.flip(0))
        codes, scales = qo.quantise(y, bits)
        got_s = cache.scales[0, 0, :, 0, j].cpu().numpy()
        np.testing.assert_array_equal(got_s, scales)
        fine = np.repeat(scales != 255, 32, -1)
        got = qo.unpack(t[0, 0, :, 0].cpu().numpy(), bits)
        np.testing.assert_array_equal(got[fine], codes[fine])
        back = f64((K, V)[j][0, 0, :, 0])
        want = qo.values(codes, scales, bits)
        assert np.isnan(back[~fine]).all()
        np.testing.assert_array_equal(back[fine], want[fine])
        assert np.isfinite(back[fine]).all()


@pytest.mark.parametrize("bits", BITS)
def test_every_bf16_value(dev, bits):
    """As a group's largest magnitude, its neighbours of all smaller magnitudes; as they come
    (groups of one exponent); in no order."""
    announce(f"every bf16, {bits} bits")
    x = torch.arange(65536).to(torch.int32).to(torch.int16).view(torch.bfloat16)
    g = torch.Generator().manual_seed(1)
    top = x.view(-1, 1)                                   # one group each
    u = torch.rand((65536, 31), generator=g)
    rest = (top.float() * u * torch.randint(-1, 2, u.shape, generator=g)).to(torch.bfloat16)
    rest = torch.where(rest.abs() <= top.abs(), rest, torch.zeros_like(rest))
    groups = torch.cat([rest, top], 1)
    groups = torch.gather(groups, 1, torch.rand((65536, 32), generator=g).argsort(1))
    written(groups.reshape(-1, D), bits, dev)
    written(x.view(-1, D), bits, dev)
    written(x[torch.randperm(65536, generator=g)].view(-1, D), bits, dev)
    written(torch.cat([groups[:, 5:], top, rest[:, :4]], 1)[:, :32].reshape(-1, D), bits, dev)


@pytest.mark.parametrize("bits", BITS)
def test_every_border(dev, bits):
    """Values on and next to the borders between elements, of both signs, by scales from
    the least to the largest."""
    announce(f"borders, {bits} bits")
    grid = qo.elements(bits)[:2 ** (bits - 1)]
    grid = grid[np.isfinite(grid)]
    top = grid[-1]
    mid = (grid[1:] + grid[:-1]) / 2
    y = np.concatenate([grid, mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -8)])
    y = np.concatenate([y, -y])
    y = np.pad(y, (0, -len(y) % 31)).reshape(-1, 31)
    y = np.concatenate([y, np.full((len(y), 1), top)], 1)
    for e in (-140, -118, -111, -60, 0, 1, 60, 110, 118, 119 if bits == 8 else 125):
        x = torch.tensor(y * 2.0 ** e).to(torch.bfloat16)
        x = torch.cat([x, x[:(-len(x)) % 4]]) if len(x) % 4 else x
        written(x.reshape(-1, D), bits, dev)


@pytest.mark.parametrize("bits", BITS)
def test_every_byte_reads_back(dev, bits):
    """All elements by all scales, also those that are never written."""
    announce(f"every byte, {bits} bits")
    rows = 256 * 256 * 8 // bits // D * 2
    k = torch.arange(256, dtype=torch.int32).to(torch.uint8).repeat(rows * D * bits // 8 // 256)
    k = k.view(1, 1, rows, 1, -1)
    s = (torch.arange(rows * 8) % 256).to(torch.uint8).view(1, 1, rows, 1, 2, 4)
    g = torch.Generator().manual_seed(2)
    v = torch.randint(0, 256, k.shape, generator=g, dtype=torch.uint8)
    cache = spec.QuantCache.of(k.to(dev), v.to(dev), s.to(dev))
    got = spec.quant_read(cache, i32([rows], dev))
    for a, b in zip(got, read(cache)):
        a = f64(a)
        # Outside bf16, which no written row is: 448 2^127 is an infinity, and 2^-9 2^-127,
        # under half of the least bf16 number 2^-133, rounds to 0.
        b = f64(torch.tensor(b).float().to(torch.bfloat16))
        np.testing.assert_array_equal(a, b)


APPEND = [
    # layers, B, L_cap, H_kv, T, pos, n_new
    (1, 1, 1, 1, 1, [0], None),
    (2, 3, 40, 2, 5, [0, 35, 17], [5, 5, 0]),
    (2, 4, 40, 3, 7, [-3, 36, -9, 2 ** 31 - 1], [7, 7, 7, 7]),      # outside in part or whole
    (1, 4, 100, 8, 64, [36, 0, 37, -64], [-5, 1000, 64, 63]),       # clamped numbers
    (3, 2, 513, 5, 300, [213, 1], None),
    (1, 2, 33, 16, 33, [0, -2 ** 31], None),
]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"n{c[0]}_b{c[1]}_h{c[3]}_t{c[4]}")
def test_append(dev, case, bits):
    n, B, cap, H_kv, T, pos, n_new = case
    announce(f"append {case} {bits}")
    for strided in (False, True):
        cache = held((n, B, cap, H_kv), 3, bits, dev)
        if strided:   # sequences and layers apart, and bytes between them that stay
            wide = held((n + 1, B + 2, cap + 2, H_kv), 4, bits, dev)
            for t, w in zip((cache.k, cache.v, cache.scales), (wide.k, wide.v, wide.scales)):
                w[:n, 1:B + 1, :cap] = t
            before = [t.clone() for t in (wide.k, wide.v, wide.scales)]
            cache = spec.QuantCache.of(*(t[:n, 1:B + 1, :cap]
                                         for t in (wide.k, wide.v, wide.scales)))
        k_new, v_new = (normal((n, B, T, H_kv, D), 5 + i, dev, 3.0) for i in range(2))
        want = [t.cpu().numpy().copy() for t in (cache.k, cache.v, cache.scales)]
        for b in range(B):
            rows = T if n_new is None else max(0, min(n_new[b], T))
            for i in range(rows):
                t = pos[b] + i
                if 0 <= t < cap:
                    for j, new in enumerate((k_new, v_new)):
                        codes, scales = qo.quantise(f64(new[:, b, i]), bits)
                        want[j][:, b, t] = qo.pack(codes, bits)
                        want[2][:, b, t, :, j] = scales
        spec.quant_append(cache, k_new, v_new, i32(pos, dev),
                          n_new=None if n_new is None else i32(n_new, dev))
        for t, w in zip((cache.k, cache.v, cache.scales), want):
            np.testing.assert_array_equal(t.cpu().numpy(), w)
        if strided:
            for t, w in zip((wide.k, wide.v, wide.scales), before):
                t[:n, 1:B + 1, :cap] = 0
                w[:n, 1:B + 1, :cap] = 0
                assert torch.equal(t, w)


# ------------------------------------------------------------------ read back

READ = [
    # layers, B, L_cap, H_kv, k_max, n_sets, counts
    (1, 1, 1, 1, 1, 1, [1]),
    (2, 3, 50, 3, 17, 1, [17, 0, 5]),
    (2, 3, 50, 3, 17, 3, [17, -4, 99]),
    (1, 2, 300, 8, 300, 8, [300, 257]),
    (3, 5, 129, 4, 64, 1, [64, 63, 1, 0, 33]),
]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("case", READ, ids=lambda c: f"n{c[0]}_b{c[1]}_h{c[3]}_k{c[4]}_s{c[5]}")
def test_read(dev, case, bits):
    n, B, cap, H_kv, k_max, sets, counts = case
    announce(f"read {case} {bits}")
    cache = held((n, B, cap, H_kv), 11, bits, dev)
    K, V = read(cache)
    rng = np.random.default_rng(12)
    idx = rng.integers(-3, cap + 3, (B, sets, k_max), dtype=np.int32)   # any order, twice, outside
    at = np.clip(idx, 0, cap - 1)
    ix = i32(idx if sets > 1 else idx[:, 0], dev)
    for given in (ix, None):
        for own_out in (False, True):
            out = None
            if own_out:
                out = tuple(torch.full((n, B, k_max, H_kv, D), 7.0, dtype=torch.bfloat16,
                                       device=dev) for _ in range(2))
            if given is None and not own_out:
                got = spec.quant_read(cache, i32(counts, dev))
                assert got[0].shape[2] == cap
            else:
                got = spec.quant_read(cache, i32(counts, dev), idx=given, out=out)
            assert not own_out or (got[0] is out[0] and got[1] is out[1])
            rows = got[0].shape[2]
            for g, src in zip(got, (K, V)):
                g = f64(g)
                for b in range(B):
                    m = max(0, min(counts[b], rows))
                    assert (g[:, b, m:] == (7.0 if own_out else 0.0)).all()
                    for h in range(H_kv):
                        t = np.arange(m) if given is None else at[b, h % sets if sets > 1 else 0,
                                                                  :m]
                        np.testing.assert_array_equal(g[:, b, :m, h], src[:, b, t, h])


# ------------------------------------------------------------------ decode attention

DECODE = [
    # layers, H_q, H_kv, L_cap, lens, window (None: all), sinks
    (1, 1, 1, 1, [1, 0], None, 0),
    (1, 8, 8, 70, [0, 1, 2, 31, 32, 33, 64, 65, 70, -3, 99], None, 0),
    (2, 12, 4, 700, [700, 699, 1], 100, 4),
    (1, 6, 2, 300, [300, 64, 5], 16, 300),
    (2, 28, 4, 1000, [1000, 517], None, 0),
    (1, 32, 8, 4096, [4096], None, 0),
    (1, 16, 1, 5000, [5000, 3], None, 0),
    (1, 34, 2, 260, [260, 130], 77, 1),                 # 17 query heads each
    (1, 48, 2, 515, [515, 96], None, 0),                # 24
    (1, 128, 1, 300, [299, 33], None, 0),
    (3, 10, 5, 333, [333, 32, 100], 50, 0),             # five heads: one at a time
    (4, 32, 8, 2300, [2300 - 97 * b for b in range(16)], 1024, 4),
    (32, 8, 2, 96, [96 - b for b in range(32)], None, 0),
    (1, 8, 8, 20011, [20011], 8000, 1),
]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_l{c[3]}_w{c[5]}")
def test_decode(dev, case, bits):
    n, H_q, H_kv, cap, lens, window, sinks = case
    announce(f"decode {case} {bits}")
    B, G = len(lens), H_q // H_kv
    cache = held((n, B, cap, H_kv), 21, bits, dev, hidden=lens)
    q = normal((n, B, H_q, D), 22, dev)
    out, lse = spec.quant_decode_attn(q, cache, i32(lens, dev), window=window, n_sink=sinks)
    assert torch.isfinite(out).all()
    K, V = read(cache)
    some = [(0, 0, 0), (n - 1, B - 1, H_kv - 1), (n // 2, B // 2, H_kv // 2)]
    some += [(0, b, b % H_kv) for b in range(B)]
    for layer, b, g in sorted(set(some)):
        heads = slice(g * G, (g + 1) * G)
        rows = seen(min(lens[b], cap), cap if window is None else window, sinks)
        compare((layer, b, g), f64(out[layer, b, heads]), f64(lse[layer, b, heads]),
                f64(q[layer, b, heads]), K[layer, b, rows, g], V[layer, b, rows, g])


SPARSE = [
    # layers, H_q, H_kv, L_cap, k_max, n_sets, counts
    (1, 1, 1, 1, 1, 1, [1, 0]),
    (1, 8, 8, 70, 70, 1, [0, 1, 2, 31, 32, 33, 64, 65, 70, -3, 99]),
    (2, 12, 4, 700, 100, 4, [100, 99, 1]),
    (2, 28, 4, 3000, 517, 1, [517, 500]),
    (1, 32, 8, 4096, 512, 1, [512]),
    (1, 16, 1, 5000, 2048, 1, [2048, 3]),
    (1, 34, 2, 260, 33, 2, [33, 20]),
    (1, 128, 1, 300, 40, 1, [40, 33]),
    (3, 10, 5, 333, 64, 5, [64, 32, 50]),
    (4, 32, 8, 2300, 600, 8, [600 - 31 * b for b in range(16)]),
    (32, 8, 2, 96, 50, 1, [50 - b for b in range(32)]),
]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("case", SPARSE, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_k{c[4]}_s{c[5]}")
def test_sparse(dev, case, bits):
    n, H_q, H_kv, cap, k_max, sets, counts = case
    announce(f"sparse {case} {bits}")
    B, G = len(counts), H_q // H_kv
    cache = held((n, B, cap, H_kv), 31, bits, dev)
    q = normal((n, B, H_q, D), 32, dev)
    rng = np.random.default_rng(33)
    idx = np.full((B, sets, k_max), -7, dtype=np.int32)
    for b, s in itertools.product(range(B), range(sets)):
        m = max(0, min(counts[b], k_max))
        idx[b, s, :m] = np.sort(rng.choice(cap, m, replace=False)) if b % 2 == 0 else \
            rng.integers(0, cap, m)                  # also in no order, an index twice
        if m > 2 and b % 3 == 1:
            idx[b, s, :2] = (cap + 5, -1)            # clamped
    # rows that no query sees are NaN
    at = np.clip(idx, 0, cap - 1)
    for b, g in itertools.product(range(B), range(H_kv)):
        m = max(0, min(counts[b], k_max))
        hide = np.setdiff1d(np.arange(cap), at[b, g if sets > 1 else 0, :m])
        cache.scales[:, b, torch.as_tensor(hide, device=dev), g] = 255
    out, lse = spec.quant_sparse_decode_attn(q, cache, i32(counts, dev),
                                             i32(idx if sets > 1 else idx[:, 0], dev))
    assert torch.isfinite(out).all()
    K, V = read(cache)
    some = [(0, 0, 0), (n - 1, B - 1, H_kv - 1), (n // 2, B // 2, H_kv // 2)]
    some += [(0, b, b % H_kv) for b in range(B)]
    for layer, b, g in sorted(set(some)):
        heads = slice(g * G, (g + 1) * G)
        rows = at[b, g if sets > 1 else 0, :max(0, min(counts[b], k_max))]
        compare((layer, b, g), f64(out[layer, b, heads]), f64(lse[layer, b, heads]),
                f64(q[layer, b, heads]), K[layer, b, rows, g], V[layer, b, rows, g])
