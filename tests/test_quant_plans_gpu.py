"""Decode attention over caches in 4 and 8 bits at shapes that take every way of dividing a
launch: 4 and 8 wavefronts a workgroup, 1 to 8 units side by side, in parts and not, one
KV head or two to a wavefront, by 4, 8 and 16 columns of query heads."""
import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from tests.gpu_helpers import announce, f64, need_gpu
from tests.quant_helpers import D, compare, held, i32, normal, read_head

pytestmark = pytest.mark.gpu

# layers, sequences, tokens, KV heads
SHAPES = [(1, 1, 200, 1), (1, 1, 200, 3), (1, 1, 200, 8), (1, 3, 4096, 3), (1, 2, 20011, 1),
          (16, 3, 700, 2), (1, 32, 1000, 2), (4, 64, 333, 4), (16, 3, 1000, 4), (1, 32, 1500, 8),
          (4, 64, 256, 8), (32, 3, 333, 8), (4, 64, 96, 8), (8, 3, 8192, 8), (1, 1, 65536, 8),
          (1, 16, 700, 8)]


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


@pytest.mark.parametrize("bits", (4, 8))
@pytest.mark.parametrize("G", (2, 6, 16))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n{}_b{}_l{}_h{}".format(*s))
def test_plans(dev, shape, G, bits):
    check_plan(dev, shape, G, bits)


@pytest.mark.parametrize("bits", (4, 8))
@pytest.mark.parametrize("G", (1, 17, 20, 48))
@pytest.mark.parametrize("shape", [(1, 1, 200, 3), (1, 16, 700, 8), (4, 64, 96, 4), (8, 3, 8192, 2)],
                         ids=lambda s: "n{}_b{}_l{}_h{}".format(*s))
def test_column_groups(dev, shape, G, bits):
    """One query head per KV head, and several groups of them: as many as there are, where
    their number has no divisor up to 16."""
    check_plan(dev, shape, G, bits)


def check_plan(dev, shape, G, bits):
    n, B, L, H_kv = shape
    announce(f"plans {shape} {G} {bits}")
    cap = L + 5
    cache = held((1, 1, cap, H_kv), 301, bits, dev)
    if n * B > 1:      # every layer and sequence its own: rolled along the tokens
        r = [torch.stack([torch.stack([t[0, 0].roll(7 * l + 3 * b, 0) for b in range(B)])
                          for l in range(n)]) for t in (cache.k, cache.v, cache.scales)]
        cache = spec.QuantCache.of(*r)
    q = normal((n, B, G * H_kv, D), 302, dev)
    rng = np.random.default_rng(303)
    lens = rng.integers(1, L + 1, B)
    lens[0] = L
    lens[-1] = L if B == 1 else 0
    idx = torch.full((B, 1, L), -1, dtype=torch.int32)
    for b, m in enumerate(lens):
        idx[b, 0, :m] = torch.as_tensor(np.sort(rng.choice(cap, m, replace=False)))
    idx = idx[:, 0].contiguous().to(dev)
    ln = i32(lens, dev)
    wide = spec.quant_decode_attn(q, cache, ln)
    win = spec.quant_decode_attn(q, cache, ln, window=max(1, L // 2), n_sink=33)
    sel = spec.quant_sparse_decode_attn(q, cache, ln, idx)
    for t in (*wide, *win, *sel):
        assert not torch.isnan(t).any()
    some = {(0, 0, 0), (n - 1, B - 1, H_kv - 1), (n // 2, B // 2, H_kv // 2),
            (0, B // 3, H_kv - 1)}
    for layer, b, g in sorted(some):
        K, V = read_head(cache, layer, b, g)
        m, hs = int(lens[b]), slice(g * G, (g + 1) * G)
        t = np.arange(m)
        for what, (out, lse), rows in (
                ("all", wide, t), ("window", win, t[(t < 33) | (t > m - 1 - max(1, L // 2))]),
                ("selected", sel, idx[b, :m].cpu().numpy())):
            compare((what, layer, b, g), f64(out[layer, b, hs]), f64(lse[layer, b, hs]),
                    f64(q[layer, b, hs]), K[rows], V[rows])
