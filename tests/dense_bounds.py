"""Inputs whose attention is known exactly, and error bounds from a query's own logits, for
the entry points over caches that are read in full.  U = 2^-24: half a step of fp32,
relative.

Counted tokens: keys of zeros, so that every visible token weighs 1, and rows of V with one
value each, a(t) in dimension (t + shift) mod 128.  An output is then sum a(t) / n over the
visible tokens of its dimension: the sums are whole numbers of eighths and exact in fp32,
n and 1 / n (one rounding), and the product of the two takes another, so that an fp32 output
is off by 2 U of itself at most (4 U are allowed, 2^-8 more where it is rounded to bf16), and
a token too few or too many changes it by one part in its count.  The log-sum-exp is log(n):
a logarithm (2 U) and a product with ln 2 (2 U): 6 U are allowed; a token is 1 / n of it.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
D = 128
SCALE = 1.0 / math.sqrt(D)


# ------------------------------------------------------------------ counted tokens

def amplitude(t):
    """a(t): tokens 128 apart, which share a dimension, differ (t: an array or tensor)."""
    return 1.0 + (t // D % 7) / 8.0


def shift_of(layer, b, g):
    """Dimensions by which the tokens of a layer, sequence and KV head are moved on."""
    return (5 * layer + 11 * b + 37 * g) % D


def counted_values(n, B, L, H_kv, device):
    """V [n][B][L][H_kv][D] in bf16 (a shared prefix: B = 1)."""
    t = torch.arange(L, device=device)
    V = torch.zeros((n, B, L, H_kv, D), dtype=torch.bfloat16, device=device)
    a = amplitude(t).to(torch.bfloat16)
    for layer in range(n):
        for b in range(B):
            for g in range(H_kv):
                V[layer, b, t, g, (t + shift_of(layer, b, g)) % D] = a
    return V


def counts_table(L, device):
    """[L + 1][D] float64: sums of a(t) over the tokens before t, by dimension, shift 0."""
    t = torch.arange(L, device=device)
    x = torch.zeros((L + 1, D), dtype=torch.float64, device=device)
    x[t + 1, t % D] = amplitude(t).double()
    return x.cumsum(0)


def window_ranges(p, window, n_sink):
    """Of queries at positions p (a tensor): s, lo, hi; tokens [0, s) and [lo, hi) are seen."""
    hi = (p + 1).clamp(min=0)
    s = hi.clamp(max=n_sink)
    return s, torch.maximum(p - window + 1, s), hi


def counted_window(table, p, window, n_sink):
    """Outputs [len(p)][D] at shift 0 and numbers of visible tokens."""
    s, lo, hi = window_ranges(p, window, n_sink)
    n = s + hi - lo
    return (table[s] + table[hi] - table[lo]) / n.clamp(min=1)[:, None], n


def lse_of(n):
    return torch.log(n.double())      # of none: -inf


# ------------------------------------------------------------------ bounds of any inputs

def attend(q, k, v, parts, scale=SCALE):
    """One query [D] over rows k, v [n][D] (float64): output, log-sum-exp, and how far an
    fp32 pass may be from them.

    A logit is D exact products added in fp32.  Its roundings are U of the partial sums, which
    walk from 0 to the logit: a sum of independent errors of standard deviation
    U sqrt(D) / sqrt(6) |q k|_2 for a walk without drift and U sqrt(D) / 3 |q.k| for one with,
    of which 6 are allowed (the squares' sums: D / 2 and D / 3 of the final square, and the
    roundings are uniform, 1 / sqrt(3)).  Scaling and the exponential's argument take 5 U
    |logit| more, the exponential 4 U.  A weight's relative error e_t moves the output by p_t
    (v_t - out), the log-sum-exp by p_t: both are added up in full.  Sums of n terms are off by
    (8 + sqrt(n)) U of the sum of absolute values (a lane adds far fewer than n in turn).
    Weights that enter the products as `parts` bf16 numbers are off by 2^-8, 2^-17 or 2^-26 of
    themselves independently: 4 of |p v|_2.  Rounding the output is left to the caller."""
    s = scale * (k @ q)
    top = s.max()
    w = np.exp(s - top)
    z = w.sum()
    p = w / z
    out, lse = p @ v, top + math.log(z)
    qk = np.sqrt((k * k) @ (q * q))
    e = 2.5 * U * math.sqrt(D) * scale * (qk + np.abs(k @ q)) + 5 * U * np.abs(s) + 4 * U
    n = len(s)
    sums = (8 + math.sqrt(n)) * U
    part = {1: 2.0 ** -8, 2: 2.0 ** -17, 3: 2.0 ** -26}[parts]
    tol = ((p * e) @ np.abs(v - out) + sums * (p @ np.abs(v) + np.abs(out))
           + 4 * part * np.sqrt((p * p) @ (v * v)) + 1e-30)
    return out, lse, tol, (p * e).sum() + sums + 4 * U * (abs(top) + abs(lse) + 1)


# ------------------------------------------------------------------ weights of known low bits

def bf16(x):
    return torch.tensor(x, dtype=torch.float64).to(torch.bfloat16).double().numpy()


def left_out(w, parts):
    """What is left of w after it has been taken apart into `parts` bf16 numbers, relatively."""
    r = np.asarray(np.float32(w), dtype=np.float64)
    rest = r.copy()
    for _ in range(parts):
        rest = rest - bf16(rest)
    return np.abs(rest) / r


def two_level_queries(n_heads):
    """First elements x of queries whose logit over a key of -4 gives a weight w = exp(-4 x
    SCALE) of which two bf16 numbers leave out 40 to 120 U: (x, w)."""
    x = bf16(1.0 + np.arange(128) / 128.0)
    w = np.exp(-4.0 * x * SCALE)
    r = left_out(w, 2) / U
    good = (r > 40) & (r < 120)
    x, w = x[good], w[good]
    assert len(x) >= 8
    return np.resize(x, n_heads), np.resize(w, n_heads)


def two_level_cache(n, B, L, H_kv, device):
    """Even tokens have keys of 0 (weight 1) and V of 1 in dimension t / 2 mod 64, odd ones
    first elements of -4 (weight w) and V of 1 in dimension 64 + t / 2 mod 64."""
    K = torch.zeros((n, B, L, H_kv, D), dtype=torch.bfloat16, device=device)
    V = torch.zeros_like(K)
    t = torch.arange(L, device=device)
    K[:, :, 1::2, :, 0] = -4.0
    V[:, :, t, :, 64 * (t % 2) + t // 2 % 64] = 1.0
    return K, V


def two_level_tolerance(tokens_per_dim, parts):
    """Of out[64 + j] / out[j] against w, relatively (as many tokens in both).  |log2 w| < 1:
    4 roundings of the argument are 4 U ln 2, the exponential 2 U, `parts` products a token
    added in turn a U each, the division by the common sum 2 U: (7 + parts tokens) U, and 4
    more; and what two numbers leave out."""
    return (11 + parts * tokens_per_dim) * U + (2.0 ** -17 if parts == 2 else 0.0)
