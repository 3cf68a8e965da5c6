"""What the tests of the caches held in 4 or 8 bits share."""
import math

import numpy as np
import torch

import paper_2512_00722_amd as spec
from oracle import quant_oracle as qo
from tests import dense_bounds as db

D = 128


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def normal(shape, seed, dev, sd=1.0):
    g = torch.Generator().manual_seed(seed)
    return (sd * torch.randn(shape, generator=g)).to(torch.bfloat16).to(dev)


def held(shape, seed, bits, dev, hidden=None):
    """A cache [n, B, L, H_kv] of random elements with scales of 2^-3 .. 2^1 (8 bits: 2^-9 ..
    2^-5), made on the host; the rows behind `hidden` [B] tokens are NaN."""
    n, B, L, H_kv = shape
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randint(0, 256, (*shape, D * bits // 8), generator=g, dtype=torch.uint8)
            for _ in range(2))
    if bits == 8:    # no NaN elements
        k, v = (torch.where((t & 127) == 127, t - 1, t) for t in (k, v))
    low = 124 if bits == 4 else 118
    s = torch.randint(low, low + 5, (*shape, 2, 4), generator=g, dtype=torch.uint8)
    if hidden is not None:
        for b, m in enumerate(hidden):
            s[:, b, max(0, min(m, L)):] = 255
    return spec.QuantCache.of(k.to(dev), v.to(dev), s.to(dev))


def read(cache):
    """K, V [n, B, L, H_kv, D] float64 of a cache, by the oracle."""
    s = cache.scales.cpu().numpy()
    return tuple(qo.values(qo.unpack(t.cpu().numpy(), cache.bits), s[..., j, :], cache.bits)
                 for j, t in enumerate((cache.k, cache.v)))


def seen(length, window, n_sink):
    t = np.arange(max(length, 0))
    return t[(t < n_sink) | (t > length - 1 - window)]


def compare(what, out, lse, q, k, v):
    """out, lse [G][D], [G] of queries q [G][D] over rows k, v [n][D] (all float64)."""
    for h in range(q.shape[0]):
        if len(k) == 0:
            assert (out[h] == 0).all() and lse[h] == -math.inf, (what, h)
            continue
        want, wlse, tol, tol_lse = db.attend(q[h], k, v, 3)
        tol = tol + db.U * np.abs(want)      # the output's own rounding
        err = np.abs(out[h] - want)
        assert (err <= tol).all(), (what, h, float((err / tol).max()))
        assert abs(lse[h] - wlse) <= tol_lse, (what, h, abs(lse[h] - wlse) / tol_lse)


def read_head(cache, layer, b, g):
    """K, V [L, D] float64 of one KV head, by the oracle."""
    s = cache.scales[layer, b, :, g].cpu().numpy()
    return tuple(qo.values(qo.unpack(t[layer, b, :, g].cpu().numpy(), cache.bits), s[:, j],
                           cache.bits) for j, t in enumerate((cache.k, cache.v)))
