"""The entry points over caches that are read in full, where arguments share memory and
where logits of -inf meet values that are not finite.  Tolerances as in
test_dense_gpu.py."""
import math

import numpy as np
import pytest
import torch

import paper_2512_00722_amd as spec
from oracle import dense_oracle
from tests.gpu_helpers import announce, f64
from tests.test_dense_gpu import (D, SCALE, U, bounded, cache, check, dev, evict_reference, finite,
                                  i32, normal, same_bits, weight_error)

pytestmark = pytest.mark.gpu
assert dev  # the fixture


# ------------------------------------------------------------------ eviction

@pytest.mark.parametrize("T,cap", [(30, 100), (40, 100), (30, 40000)])
@pytest.mark.parametrize("alias", ["n_new", "keep"])
def test_evict_arguments_in_the_counts(dev, T, cap, alias):
    """The new rows, or the budgets, read from the tensor of the counts, which the call
    rewrites."""
    announce(f"evict {alias} in the counts, {T} {cap}")
    n, B, H_kv = 2, 3, 2
    counts = [20, cap, 25] if alias == "n_new" else [20, 60, 0]
    rows = [min(c, T) for c in counts] if alias == "n_new" else [T, 7, 2]
    keep = [35, 60, 40] if alias == "n_new" else counts
    x = bounded(n, B, H_kv, H_kv, cap, 301, dev)
    x[3][:, 0] = torch.randperm(cap, generator=torch.Generator().manual_seed(302)).int().to(dev)
    x[3][:, 0, :, :20] = torch.arange(180, 200, dtype=torch.int32).flip(0).to(dev)
    pos = [200, 3 * cap, 50]
    k_new, v_new = (normal((n, B, T, H_kv, D), 303 + i, dev) for i in range(2))
    *want, after = evict_reference(x, H_kv, counts, keep, pos, rows, k_new, v_new, 25, 2)
    c = i32(counts, dev)
    spec.evict(*x, c, c if alias == "keep" else i32(keep, dev), i32(pos, dev), k_new=k_new,
               v_new=v_new, n_new=c if alias == "n_new" else i32(rows, dev), n_recent=25, n_sink=2)
    torch.cuda.synchronize()
    assert c.tolist() == after
    for got, ref, nm in zip(x, want, ("K", "V", "weights", "tokens")):
        assert same_bits(got, ref), nm


# ------------------------------------------------------------------ logits of -inf

DEAD = [
    # layers, H_q, H_kv, cap, tokens whose logits are -inf, T of the chunk
    (1, 8, 2, 300, slice(0, 300), 40),           # all
    (1, 8, 2, 300, slice(3, 290), 40),
    (1, 32, 8, 3000, slice(0, 2900), 8),         # whole parts of a divided cache
    (1, 4, 1, 20000, slice(100, 19000), 3),
    (1, 4, 1, 20000, slice(0, 20000), 3),
    (1, 32, 2, 600, slice(0, 550), 200),         # every row tile
    (1, 128, 2, 500, slice(0, 200), 300),
    (1, 8, 8, 40, slice(0, 39), 2),
    (16, 32, 8, 130, slice(0, 129), 2),          # accumulated weights in LDS
]


@pytest.mark.parametrize("case", DEAD, ids=lambda c: f"n{c[0]}_h{c[1]}_{c[2]}_l{c[3]}_{c[4].start}_{c[4].stop}")
@pytest.mark.parametrize("odd", [0.5, math.nan, math.inf], ids=["finite", "nan", "inf"])
def test_tokens_whose_logits_are_minus_infinity(dev, case, odd):
    """They weigh nothing, whatever their rows of V hold; where there are no others a
    query gets 0 and -inf."""
    n, H_q, H_kv, cap, dead, T = case
    announce(f"-inf {case} {odd}")
    B, G, P = 2, H_q // H_kv, 600
    K, V = cache(n, B, cap, H_kv, 311, dev)
    Kp, Vp = (normal((n, P, H_kv, D), 313 + i, dev) for i in range(2))
    q, qc = normal((n, B, H_q, D), 315, dev), normal((n, B, T, H_q, D), 316, dev)
    for t in (q, qc):
        t[..., 0] = t[..., 0].abs() + 0.125
    for x, k, at in ((K, V, dead), (Kp, Vp, slice(40, P))):
        x[..., at, :, 0] = -math.inf
        k[..., at, :, 5] = odd
    lens = i32([cap, cap], dev)
    l, b, g = n - 1, 1, H_kv - 1
    heads = slice(g * G, (g + 1) * G)
    live = [t for t in range(cap) if not dead.start <= t < dead.stop]
    kk, vv = f64(K[l, b, live, g:g + 1]), f64(V[l, b, live, g:g + 1])
    qq = f64(q[l, b, heads])
    kp, vp = f64(Kp[l, :40, g:g + 1]), f64(Vp[l, :40, g:g + 1])

    def compare(what, out, lse, ks, vs):
        want, wlse, _ = dense_oracle.accumulate(qq, ks, vs, 1, SCALE)
        spread, _, _ = dense_oracle.accumulate(qq, ks, np.abs(vs), 1, SCALE)
        e = weight_error(qq, ks, cap + P)
        check(out.cpu(), want, 2 * e * spread + 1e-30, (what, "out"))
        check(lse.cpu(), wlse, e + 16 * U * np.abs(finite(wlse)), (what, "lse"))

    out, lse = spec.window_decode_attn(q, K, V, lens, cap)
    compare("window decode", out[l, b, heads], lse[l, b, heads], kk, vv)
    w = torch.zeros((n, B, H_kv, cap), device=dev)
    out, lse = spec.accum_decode_attn(q, K, V, lens, w)
    compare("accum", out[l, b, heads], lse[l, b, heads], kk, vv)
    assert not w[..., dead].any() and torch.isfinite(w).all()
    assert abs(float(w[l, b, g].sum()) - (G if live else 0)) <= G * 2.0 ** -10
    out, lse = spec.prefix_decode_attn(q, Kp, Vp, K, V, lens)
    compare("prefix", out[l, b, heads], lse[l, b, heads], np.concatenate([kp, kk]),
            np.concatenate([vp, vv]))
    out, lse = spec.window_attn(qc, K, V, lens, cap)
    for i in {0, T // 2, T - 1}:
        seen = [t for t in live if t <= cap - T + i]
        qi = f64(qc[l, b, i, heads])
        ks, vs = f64(K[l, b, seen, g:g + 1]), f64(V[l, b, seen, g:g + 1])
        want, wlse, _ = dense_oracle.accumulate(qi, ks, vs, 1, SCALE)
        spread, _, _ = dense_oracle.accumulate(qi, ks, np.abs(vs), 1, SCALE)
        e = weight_error(qi, ks, cap)
        check(f64(out[l, b, i, heads]), want,
              (2 * e + 2.0 ** -8) * spread + 2.0 ** -8 * np.abs(want) + 1e-30, ("chunk", i))
        check(lse[l, b, i, heads].cpu(), wlse, e + 16 * U * np.abs(finite(wlse)), ("chunk lse", i))
