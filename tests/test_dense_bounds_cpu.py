"""That the exact inputs and the bounds of dense_bounds hold for an fp32 pass and show the
mistakes they are for: planted here, on the CPU, in emulated results."""
import math

import numpy as np
import pytest
import torch

from oracle import dense_oracle
from tests import dense_bounds as db
from tests.dense_bounds import D, SCALE, U


def rng_bf16(shape, seed, sd=1.0):
    g = torch.Generator().manual_seed(seed)
    return (sd * torch.randn(shape, generator=g)).to(torch.bfloat16).double().numpy()


def emulate(q, k, v, parts, tile=32, skip=()):
    """An fp32 pass with a running maximum, weights as `parts` bf16 numbers."""
    f = np.float32
    keep = np.array([t for t in range(len(k)) if t not in set(skip)])
    m, z, acc = f(-np.inf), f(0), np.zeros(D, f)
    for t0 in range(0, len(keep), tile):
        t = keep[t0:t0 + tile]
        x = (k[t].astype(f) @ q.astype(f)) * f(SCALE * math.log2(math.e))
        mn = max(m, x.max())
        a = f(np.exp2(f(m - mn))) if m > -np.inf else f(0)
        p = np.exp2(x - mn).astype(f)
        m, z, acc = mn, f(z * a + p.sum(dtype=f)), (acc * a).astype(f)
        rest = p.astype(np.float64)
        for _ in range(parts):
            b = db.bf16(rest)
            acc = (acc + b.astype(f) @ v[t].astype(f)).astype(f)
            rest = rest - b
    return acc.astype(np.float64) / float(z), float(m) * math.log(2) + math.log(float(z))


def inside(got, bound):
    out, lse, tol, tol_lse = bound
    return bool((np.abs(got[0] - out) <= tol).all()), abs(got[1] - lse) <= tol_lse


@pytest.mark.parametrize("n,sd", [(1, 1.0), (40, 1.0), (2000, 1.0), (20011, 1.0), (700, 4.0)])
def test_bounds_hold_for_an_fp32_pass(n, sd):
    for seed in range(4):
        q = rng_bf16((D,), seed, sd)
        k, v = (rng_bf16((n, D), 10 + seed + i) for i in range(2))
        for parts in (1, 2, 3):
            assert inside(emulate(q, k, v, parts), db.attend(q, k, v, parts)) == (True, True)


def test_bounds_show_lost_tokens_and_rounded_weights():
    """The last 11 of 20011 tokens, a tile of 64 of 32768, one of 2000, and weights in one
    number instead of two or three."""
    for n, skip in ((20011, range(20000, 20011)), (32768, range(12800, 12864)), (2000, [1999])):
        q = rng_bf16((D,), 20)
        k, v = (rng_bf16((n, D), 21 + i) for i in range(2))
        bound = db.attend(q, k, v, 2)
        assert inside(emulate(q, k, v, 2), bound) == (True, True)
        assert inside(emulate(q, k, v, 2, skip=skip), bound) == (False, False)
        # where the weights are rounded once, the log-sum-exp shows it
        assert not inside(emulate(q, k, v, 1, skip=skip), db.attend(q, k, v, 1))[1]
    q = rng_bf16((D,), 20)
    k, v = (rng_bf16((700, D), 31 + i) for i in range(2))
    assert inside(emulate(q, k, v, 1), db.attend(q, k, v, 2)) == (False, True)


def test_counted_tokens_against_the_oracle():
    L, window, sinks, T = 300, 37, 5, 40
    table = db.counts_table(L, "cpu")
    V = db.counted_values(1, 1, L, 2, "cpu")[0, 0].double().numpy()
    K = np.zeros_like(V)
    q = rng_bf16((T, 2, D), 3)
    want, n = db.counted_window(table, torch.arange(L - T, L), window, sinks)
    out, lse, _ = dense_oracle.window_attention(q, K, V, L - T, window, sinks, SCALE)
    for g in range(2):
        assert np.allclose(out[:, g], torch.roll(want, db.shift_of(0, 0, g), 1).numpy(), rtol=1e-14)
        assert np.allclose(lse[:, g], db.lse_of(n).numpy(), rtol=1e-14)
    none, n = db.counted_window(table, torch.tensor([-3, -1]), window, sinks)
    assert not none.any() and (n == 0).all() and (db.lse_of(n) == -math.inf).all()


@pytest.mark.parametrize("n", [1, 100, 8192, 20011])
def test_counted_tokens_show_every_lost_or_doubled_token(n):
    """In bf16 outputs up to 8192 tokens, in fp32 ones and the log-sum-exp at any length."""
    table = db.counts_table(n, "cpu")
    want = table[n] / n
    for t in {0, n // 2, n - 1}:
        a, at = float(db.amplitude(torch.tensor(t))), t % D
        for sign in (-1, 1):
            if n + sign == 0:
                continue
            wrong = table[n].clone()
            wrong[at] += sign * a
            wrong /= n + sign
            err = float((wrong[at] - want[at]).abs() / want[at])
            if n > 1:     # the only token twice is the same mean
                assert err > 4 * U
            if 1 < n <= 8192:
                assert err > 2.0 ** -8 + 4 * U
            assert abs(math.log(n + sign) - math.log(n)) > 6 * U * math.log(max(n, 2))
        # another token of the same dimension in its place
        if t + D < n and db.amplitude(t) != db.amplitude(t + D):
            assert abs(db.amplitude(t) - db.amplitude(t + D)) / float(table[n][at]) > 4 * U


def test_two_levels_show_the_third_number():
    """The ratio of the two levels' outputs, taken from weights in three, two and one
    numbers."""
    x, w = db.two_level_queries(8)
    for tokens in (2, 4):
        tol3, tol2 = (db.two_level_tolerance(tokens, p) for p in (3, 2))
        assert (db.left_out(w, 3) < tol3).all()
        assert (db.left_out(w, 2) > tol3).all() and (db.left_out(w, 2) < tol2).all()
        assert (db.left_out(w, 1) > tol2).any()
    K, V = db.two_level_cache(1, 1, 256, 1, "cpu")
    q = np.zeros(D)
    q[0] = x[0]
    out, _, _ = dense_oracle.attend(q, K[0, 0, :, 0].double().numpy(),
                                    V[0, 0, :, 0].double().numpy(), SCALE)
    assert np.allclose(out[64:] / out[:64], w[0], rtol=1e-14)
    got, _ = emulate(q, K[0, 0, :, 0].double().numpy(), V[0, 0, :, 0].double().numpy(), 3)
    assert (np.abs(got[64:] / got[:64] / w[0] - 1) < db.two_level_tolerance(2, 3)).all()
    got, _ = emulate(q, K[0, 0, :, 0].double().numpy(), V[0, 0, :, 0].double().numpy(), 2)
    assert (np.abs(got[64:] / got[:64] / w[0] - 1) > db.two_level_tolerance(2, 3)).all()
