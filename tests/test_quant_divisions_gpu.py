"""Decode attention over caches in 4 and 8 bits in the divisions of a launch that the shapes
of test_quant_plans_gpu.py do not have (test_quant_divisions_cpu.py compares both with what
the planner can choose)."""
import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from tests import quant_divisions as qd
from tests.gpu_helpers import announce, f64, need_gpu
from tests.quant_helpers import D, compare, held, i32, normal, read_head, seen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


@pytest.mark.parametrize("case", qd.CASES, ids=lambda c: "n{}_b{}_l{}_h{}x{}_{}bit_{}{}".format(*c))
def test_divisions(dev, case):
    announce(f"division {case}")
    n, B, L, H_kv, G, bits, kind, tokens, n_sink = case
    cache = held((1, 1, L, H_kv), 311, bits, dev)
    if n * B > 1:      # every layer and sequence its own: rolled along the tokens
        cache = spec.QuantCache.of(*(
            torch.stack([torch.stack([t[0, 0].roll(7 * l + 3 * b, 0) for b in range(B)])
                         for l in range(n)]) for t in (cache.k, cache.v, cache.scales)))
    q = normal((n, B, G * H_kv, D), 312, dev)
    rng = np.random.default_rng(313)
    most = tokens if kind == "selected" else L
    lens = rng.integers(0, most + 1, B)
    lens[0] = most
    rows = {}
    if kind == "selected":
        idx = torch.full((B, most), -1, dtype=torch.int32)
        for b, m in enumerate(lens):
            rows[b] = np.sort(rng.choice(L, m, replace=False))
            idx[b, :m] = torch.as_tensor(rows[b])
        out, lse = spec.quant_sparse_decode_attn(q, cache, i32(lens, dev), idx.to(dev))
    else:
        window = tokens if kind == "window" else None
        for b, m in enumerate(lens):
            rows[b] = seen(int(m), window or L, n_sink)
        out, lse = spec.quant_decode_attn(q, cache, i32(lens, dev), window=window, n_sink=n_sink)
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    for layer, b, g in sorted({(0, 0, 0), (n - 1, B - 1, H_kv - 1), (n // 2, B // 2, H_kv // 2),
                               (0, B // 3, H_kv - 1)}):
        K, V = read_head(cache, layer, b, g)
        hs = slice(g * G, (g + 1) * G)
        compare((layer, b, g), f64(out[layer, b, hs]), f64(lse[layer, b, hs]),
                f64(q[layer, b, hs]), K[rows[b]], V[rows[b]])
