"""The entry points over caches that are read in full, at the sizes that take
their other ways through: every row tile and split of the chunks, the
accumulated weights in LDS and in memory, every width of the eviction's plan,
and caches whose offsets pass 32 bits.  Tolerances as in test_dense_gpu.py."""
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


def some(n, k):
    """k of 0 .. n - 1, the first and the last among them."""
    return sorted({round(i * (n - 1) / max(1, k - 1)) for i in range(k)})


# ------------------------------------------------------------------ window, chunks

WINDOW = [
    # H_q, H_kv, cap, T, lens, q_lens, window, sinks
    (32, 8, 8192, 512, [8192], None, 8192, 0),               # a long cache before the chunk
    (32, 8, 4096, 4096, [4096, 4000], [4096, 3999], 4096, 4),
    (32, 8, 8192, 8192, [8192], None, 1024, 16),
    (32, 8, 2048, 2048, [2001], [2001], 2048, 0),
    (32, 8, 16384, 32, [16384], None, 16384, 1),
    (32, 8, 32768, 128, [32768], None, 32768, 0),
    (28, 4, 3001, 257, [3001, 257, 1700, 9, 0], [257, 257, 100, 9, 257], 777, 3),
    (16, 16, 4096, 2, [4096, 2, 1], None, 4096, 0),          # two rows a KV head
    (127, 1, 600, 5, [600, 4], None, 64, 2),
    (8, 8, 4096, 4096, [4096], None, 33, 0),
]


@pytest.mark.parametrize("case", WINDOW, ids=lambda c: f"h{c[0]}_{c[1]}_l{c[2]}_t{c[3]}_w{c[6]}")
def test_window(dev, case):
    H_q, H_kv, cap, T, lens, q_lens, window, sinks = case
    announce(f"window {case}")
    B, G = len(lens), H_q // H_kv
    K, V = cache(1, B, cap, H_kv, 31, dev, lens)
    q = normal((1, B, T, H_q, D), 33, dev)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:-1], 7.0, device=dev)
    spec.window_attn(q, K, V, i32(lens, dev), window, n_sink=sinks,
                     q_lens=None if q_lens is None else i32(q_lens, dev), out=out, lse=lse)
    torch.cuda.synchronize()
    rows = [T] * B if q_lens is None else q_lens
    for b in range(B):
        r = rows[b]
        assert (out[0, b, r:] == 7.0).all() and (lse[0, b, r:] == 7.0).all()
        assert not torch.isnan(out[0, b, :r]).any()
        for g in some(H_kv, 2):
            kk, vv = f64(K[0, b, :, g:g + 1]), f64(V[0, b, :, g:g + 1])
            heads = slice(g * G, (g + 1) * G)
            e = weight_error(f64(q[0, b, :r, heads]), finite(kk), cap)
            for i in some(r, 9) if r else []:
                want, wlse, spread = dense_oracle.window_attention(
                    f64(q[0, b, i:i + 1, heads]), kk, vv, lens[b] - r + i, window, sinks, SCALE)
                tol = (2 * e + 2.0 ** -8) * spread + 2.0 ** -8 * np.abs(want) + 1e-30
                check(f64(out[0, b, i:i + 1, heads]), want, tol, ("out", b, g, i))
                check(lse[0, b, i:i + 1, heads].cpu(), wlse,
                      e + 16 * U * np.abs(finite(wlse)), ("lse", b, g, i))


# ------------------------------------------------------------------ shared prefix

PREFIX = [
    # H_q, H_kv, P_cap, P, cap, lens
    (32, 8, 9000, 8999, 300, [300, 0, 17, 299] * 16),        # 256 rows
    (32, 8, 20011, None, 777, [777, 5, 400] * 5),
    (64, 8, 4097, 4096, 100, [100, 33] * 6),
    (128, 1, 3000, None, 64, [64] * 5),                      # 640 rows on one KV head
    (64, 16, 2000, 1990, 700, [700, 5, 0, 699] * 5),         # own tokens by four heads side by
    (64, 16, 1500, None, 700, [700, 31] * 6),                # side, 128 and 64 rows
    (16, 4, 900, None, 5000, [5000, 4000]),
]


@pytest.mark.parametrize("case", PREFIX, ids=lambda c: f"h{c[0]}_{c[1]}_p{c[2]}_b{len(c[5])}")
def test_prefix(dev, case):
    H_q, H_kv, P_cap, P, cap, lens = case
    announce(f"prefix {case}")
    B, G = len(lens), H_q // H_kv
    K, V = cache(1, B, cap, H_kv, 71, dev, lens)
    Kp, Vp = (normal((1, P_cap, H_kv, D), 73 + i, dev) for i in range(2))
    rows = P_cap if P is None else P
    Kp[:, rows:], Vp[:, rows:] = math.nan, math.nan
    q = normal((1, B, H_q, D), 75, dev)
    out, lse = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32(lens, dev),
                                       prefix_len=None if P is None else i32([P], dev))
    torch.cuda.synchronize()
    assert not torch.isnan(out).any()
    for g in some(H_kv, 2):
        kp, vp = f64(Kp[0, :rows, g:g + 1]), f64(Vp[0, :rows, g:g + 1])
        heads = slice(g * G, (g + 1) * G)
        for b in some(B, 6):
            qq, L = f64(q[0, b, heads]), lens[b]
            ko, vo = f64(K[0, b, :L, g:g + 1]), f64(V[0, b, :L, g:g + 1])
            want, wlse = dense_oracle.prefix_attention(qq, kp, vp, ko, vo, SCALE)
            spread, _ = dense_oracle.prefix_attention(qq, kp, np.abs(vp), ko, np.abs(vo), SCALE)
            e = weight_error(qq, np.concatenate([kp, ko]), rows + cap)
            check(out[0, b, heads].cpu(), want, 2 * e * spread + 1e-30, ("out", b, g))
            check(lse[0, b, heads].cpu(), wlse, e + 16 * U * np.abs(wlse), ("lse", b, g))


# ------------------------------------------------------------------ accumulated weights

ACCUM = [
    # layers, sequences, H_q, H_kv, cap, n_sets
    (16, 16, 9, 3, 100, 3),       # logits in LDS, a group a workgroup
    (16, 16, 9, 3, 100, 1),       # ... the sets' sums in memory
    (32, 16, 8, 2, 100, 2),       # two groups
    (32, 16, 8, 2, 100, 1),
    (16, 16, 48, 2, 90, 2),       # 24 query heads: two groups a KV head
    (16, 8, 32, 8, 130, 1),       # four groups
    (16, 8, 32, 8, 2047, 8),
    (1, 2, 4, 4, 3001, 4),        # logits in memory, in parts; a row a set
    (1, 2, 8, 2, 3001, 2),        # four
    (1, 3, 40, 2, 1500, 1),       # forty
    (1, 2, 160, 2, 700, 1),       # more than one round of rows
    (1, 1, 8, 8, 20000, 8),
    (8, 8, 64, 8, 5000, 1),       # beyond the LDS
]


@pytest.mark.parametrize("case", ACCUM, ids=lambda c: f"n{c[0]}_b{c[1]}_h{c[2]}_{c[3]}_l{c[4]}_s{c[5]}")
def test_accum(dev, case):
    n, B, H_q, H_kv, cap, n_sets = case
    announce(f"accum {case}")
    counts = [cap if b == 0 else (b * 7919) % (cap + 1) for b in range(B)]
    K, V = cache(n, B, cap, H_kv, 91, dev, counts)
    q = normal((n, B, H_q, D), 93, dev)
    w0 = torch.rand((n, B, n_sets, cap), generator=torch.Generator().manual_seed(94)).to(dev)
    w, w2 = w0.clone(), w0.clone()
    out, lse = spec.accum_decode_attn(q, K, V, i32(counts, dev), w)
    out2, none = spec.accum_decode_attn(q, K, V, i32(counts, dev), w2, with_lse=False)
    assert none is None and torch.equal(out, out2) and torch.equal(w, w2)
    assert not torch.isnan(out).any() and not torch.isnan(w).any()
    for l in some(n, 2):
        for b in some(B, 3):
            c = counts[b]
            qq, kk, vv = f64(q[l, b]), f64(K[l, b, :c]), f64(V[l, b, :c])
            want, wlse, add = dense_oracle.accumulate(qq, kk, vv, n_sets, SCALE)
            spread, _, _ = dense_oracle.accumulate(qq, kk, np.abs(vv), n_sets, SCALE)
            e = weight_error(qq, kk, cap)
            check(out[l, b].cpu(), want, 2 * e * spread + 1e-30, ("out", l, b))
            check(lse[l, b].cpu(), wlse, e + 16 * U * np.abs(finite(wlse)), ("lse", l, b))
            before = w0[l, b].double().cpu().numpy()
            # a sum over H_q / n_sets terms; each is off by 2 e, the sum by half a step a term
            sums = H_q // n_sets * U
            check(w[l, b, :, :c].cpu(), before[:, :c] + add,
                  (2 * e + 2.0 ** -19 + sums) * add + 2 * U * (before[:, :c] + add),
                  ("weights", l, b))
            assert torch.equal(w[l, b, :, c:], w0[l, b, :, c:])


# ------------------------------------------------------------------ eviction

EVICT = [
    # layers, H_kv, per head, cap, counts, keep, T, recent, sinks, weights
    (1, 2, True, 2048, [2048, 2000], [2048, 2001], 1, 100, 4, "mixed"),
    (1, 2, True, 2047, [2047, 2040], [2047, 2047], 3, 100, 4, "equal"),
    (1, 1, True, 3001, [3001, 2900], [3001, 2000], 4, 64, 4, "mixed"),
    (2, 2, False, 4096, [4096, 4096], [4096, 3000], 20, 300, 4, "mixed"),
    (1, 1, True, 8192, [8192, 8000], [8192, 8192], 300, 1000, 4, "mixed"),
    (1, 1, True, 8190, [8190, 8000], [4000, 100], 30, 10, 0, "equal"),
    (1, 1, True, 12000, [12000, 9000], [11000, 9001], 5, 500, 4, "mixed"),
    (1, 1, False, 32768, [32768, 30000], [32768, 20000], 100, 2000, 4, "mixed"),
    (1, 1, True, 32769, [32769, 30000], [30000, 30002], 2, 2000, 4, "mixed"),
    (1, 2, False, 40000, [40000, 33000], [39999, 33000], 50, 100, 4, "mixed"),
    (1, 1, True, 40000, [40000, 35000], [40000, 1], 7, 0, 0, "equal"),
    (1, 2, True, 900, [900, 895], [900, 899], 6, 30, 2, "mixed"),         # six go, and two
    (1, 2, True, 900, [900, 900], [900, 894], 6, 30, 2, "equal"),         # six, and twelve
    (1, 1, True, 4096, [4096, 4096], [1000, 4095], 0, 0, 0, "close"),     # equal but for low bits
    (1, 1, True, 700, [700, 700], [300, 100], 2, 350, 3, "inf"),          # more +inf than stay
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"l{c[3]}_t{c[6]}_{c[9]}_{c[2]}")
def test_evict(dev, case):
    n, H_kv, per_head, cap, counts, keep, T, recent, sinks, weights = case
    announce(f"evict {case}")
    B, S = len(counts), H_kv if per_head else 1
    K, V, w, t = bounded(n, B, S, H_kv, cap, 101, dev)
    if weights == "equal":
        w.fill_(0.5)
    elif weights == "close":
        w = (torch.randint(0, 1500, w.shape, generator=torch.Generator().manual_seed(5)).int()
             + 0x3f000000).view(torch.float32).to(dev)
    elif weights == "inf":
        w[..., ::2] = math.inf
    k_new = v_new = None
    if T:
        k_new, v_new = (normal((n, B, T, H_kv, D), 103 + i, dev) for i in range(2))
    pos = [cap + 3 * b for b in range(B)]
    x = (K, V, w, t)
    *want, after = evict_reference(x, S, counts, keep, pos, [T] * B, k_new, v_new, recent, sinks)
    c = i32(counts, dev)
    spec.evict(*x, c, i32(keep, dev), i32(pos, dev), k_new=k_new, v_new=v_new, n_recent=recent,
               n_sink=sinks)
    torch.cuda.synchronize()
    assert c.tolist() == after
    for got, ref, nm in zip(x, want, ("K", "V", "weights", "tokens")):
        assert same_bits(got, ref), nm


@pytest.mark.parametrize("T", [2, 40])
def test_evict_positions_in_the_counts(dev, T):
    """Until a cache is full, the tokens seen are the rows held: one tensor for both."""
    n, B, H_kv, cap = 2, 3, 2, 100
    counts = [90, 100, 0]
    x = bounded(n, B, H_kv, H_kv, cap, 231, dev)
    k_new, v_new = (normal((n, B, T, H_kv, D), 233 + i, dev) for i in range(2))
    *want, after = evict_reference(x, H_kv, counts, [cap] * B, counts, [T] * B, k_new, v_new, 8, 2)
    c = i32(counts, dev)
    spec.evict(*x, c, i32([cap] * B, dev), c, k_new=k_new, v_new=v_new, n_recent=8, n_sink=2)
    assert c.tolist() == after
    for got, ref, nm in zip(x, want, ("K", "V", "weights", "tokens")):
        assert same_bits(got, ref), nm


# ------------------------------------------------------------------ offsets past 32 bits

def test_large_offsets(dev):
    """Caches of 2.5e9 elements whose last tokens alone weigh: keys of zeros but
    for them, so that the sums are known."""
    H, cap = 64, 300011                       # cap * H * 128 > 2^31
    L, n = cap - 3, 40
    announce("large offsets")
    K, V = (torch.zeros((1, 1, cap, H, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
    K[0, 0, L:], V[0, 0, L:] = math.nan, math.nan
    K[0, 0, L - n:L], V[0, 0, L - n:L] = (normal((n, H, D), 211 + i, dev, 2.0) for i in range(2))
    q = normal((1, 1, 7, H, D), 213, dev, 2.0)
    lens = i32([L], dev)
    kk, vv = f64(K[0, 0, L - n:L]), f64(V[0, 0, L - n:L])
    qq = f64(q[0, 0])

    # the decode entry points: query 6 over all tokens; the others have logits of 0
    s = np.einsum("hd,thd->ht", qq[6], kk) * SCALE
    z = np.exp(s).sum(1) + (L - n)
    want = np.einsum("ht,thd->hd", np.exp(s), vv) / z[:, None]
    spread = np.einsum("ht,thd->hd", np.exp(s), np.abs(vv)) / z[:, None]
    e = weight_error(qq, kk, cap)
    one = q[:, :, 6].contiguous()
    w = torch.zeros((1, 1, 1, cap), device=dev)
    for what, (out, lse) in (
            ("window", spec.window_decode_attn(one, K, V, lens, cap)),
            ("accum", spec.accum_decode_attn(one, K, V, lens, w)),
            ("prefix", spec.prefix_decode_attn(one, K[0][None, 0], V[0][None, 0], K[:, :, L - 5:],
                                               V[:, :, L - 5:], i32([0], dev), prefix_len=lens))):
        check(out[0, 0].cpu(), want, 2 * e * spread + 1e-30, what)
        check(lse[0, 0].cpu(), np.log(z), e + 16 * U * np.log(z), what)
    p = np.exp(s) / z[:, None]
    check(w[0, 0, 0, L - n:L].cpu(), p.sum(0), (2 * e + 2.0 ** -19 + H * U) * p.sum(0), "weights")
    check(w[0, 0, 0, :L - n].cpu(), np.broadcast_to((1 / z).sum(), L - n),
          (2 * e + 2.0 ** -19 + H * U) * (1 / z).sum(), "weights of the others")
    assert not w[0, 0, 0, L:].any()

    # a chunk of 7 with a window of 20
    out, lse = spec.window_attn(q, K, V, lens, 20)
    wout, wlse, spread = dense_oracle.window_attention(qq, kk, vv, n - 7, 20, 0, SCALE)
    check(f64(out[0, 0]), wout, (2 * e + 2.0 ** -8) * spread + 2.0 ** -8 * np.abs(wout) + 1e-30,
          "chunk")
    check(lse[0, 0].cpu(), wlse, e + 16 * U * np.abs(wlse), "chunk lse")

    # eviction at the end of the cache: 3 rows come in, the budget is full, 3 go
    k_new, v_new = (normal((1, 1, 6, H, D), 215 + i, dev) for i in range(2))
    tok = torch.arange(cap, dtype=torch.int32, device=dev).view(1, 1, 1, cap)
    w.fill_(1.0)
    gone = [L - 1, 5, L - 30]
    w[0, 0, 0, gone] = 0.5
    c = i32([L], dev)
    spec.evict(K, V, w, tok, c, i32([cap], dev), i32([L], dev), k_new=k_new, v_new=v_new)
    slots = sorted(gone) + [L, L + 1, L + 2]
    assert c.tolist() == [cap]
    for i, t in enumerate(slots):
        assert torch.equal(K[0, 0, t], k_new[0, 0, i]) and torch.equal(V[0, 0, t], v_new[0, 0, i])
        assert int(tok[0, 0, 0, t]) == L + i and float(w[0, 0, 0, t]) == 0.0
    assert torch.equal(K[0, 0, L - 2], torch.from_numpy(kk[n - 2]).to(dev, torch.bfloat16))


# ------------------------------------------------------------------ graphs

def test_two_graphs_share_a_workspace(dev):
    """Two captured graphs and eager calls on one workspace, in turn on one stream."""
    n, B, H_q, H_kv, cap = 1, 2, 32, 8, 3000
    K, V = cache(n, B, cap, H_kv, 221, dev)
    q, qc = normal((n, B, H_q, D), 223, dev), normal((n, B, 20, H_q, D), 224, dev)
    Kp, Vp = (normal((n, 2500, H_kv, D), 225 + i, dev) for i in range(2))
    lens = i32([cap, 1700], dev)
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device=dev)
    o = [torch.zeros(q.shape, device=dev) for _ in range(3)]
    z = [torch.zeros(q.shape[:-1], device=dev) for _ in range(4)]
    oc, zc = torch.zeros_like(qc), torch.zeros(qc.shape[:-1], device=dev)
    w = torch.zeros((n, B, 1, cap), device=dev)

    def first():
        spec.window_decode_attn(q, K, V, lens, cap, out=o[0], lse=z[0], ws=ws)
        spec.accum_decode_attn(q, K, V, lens, w, out=o[1], lse=z[1], ws=ws)

    def second():
        spec.prefix_decode_attn(q, Kp, Vp, K, V, lens, out=o[2], lse=z[2], ws=ws)
        spec.window_attn(qc, K, V, lens, cap, out=oc, lse=zc, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first(), second()
    torch.cuda.current_stream().wait_stream(side)
    want = [x.clone() for x in o + z + [oc, zc]]
    graphs = []
    for f in (first, second):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            f()
    w.zero_()
    for i in range(4):
        for x in o + z + [oc, zc]:
            x.zero_()
        graphs[i % 2].replay()
        (second if i % 2 == 0 else first)()
        torch.cuda.synchronize()
        graphs[1 - i % 2].replay()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(o + z + [oc, zc], want):
            assert torch.equal(a, b), i


# ------------------------------------------------------------------ values and lengths

@pytest.mark.parametrize("B,G", [(2, 4), (12, 4), (20, 4), (40, 8)])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_prefix_odd_values(dev, B, G, odd):
    """A row of the shared V with an infinity or a NaN in one dimension: every query has
    that value there, and the other dimensions are as if it were 0."""
    P, cap = 700, 20
    lens = [cap if b % 2 else b % cap for b in range(B)]
    K, V = cache(1, B, cap, 1, 241, dev, lens)
    Kp, Vp = (normal((1, P, 1, D), 243 + i, dev) for i in range(2))
    q = normal((1, B, G, D), 245, dev)
    bad = {P - 1: 3, 100: 70, 0: 127}
    clean = Vp.clone()
    for t, dim in bad.items():
        Vp[0, t, 0, dim] = odd
        clean[0, t, 0, dim] = 0.0
    out, _ = spec.prefix_decode_attn(q, Kp, Vp, K, V, i32(lens, dev))
    kp, vp = f64(Kp[0]), f64(clean[0])
    for b in some(B, 5):
        got = out[0, b].double().cpu().numpy()
        for dim in bad.values():
            assert (np.isnan(got[:, dim]) if odd != odd else got[:, dim] == odd).all()
        ko, vo, qq = f64(K[0, b, :lens[b]]), f64(V[0, b, :lens[b]]), f64(q[0, b])
        want, _ = dense_oracle.prefix_attention(qq, kp, vp, ko, vo, SCALE)
        spread, _ = dense_oracle.prefix_attention(qq, kp, np.abs(vp), ko, np.abs(vo), SCALE)
        e = weight_error(qq, np.concatenate([kp, ko]), P + cap)
        for dim in bad.values():
            got[:, dim] = want[:, dim]
        check(got, want, 2 * e * spread + 1e-30, ("the other values", b))


def test_lengths_are_clamped(dev):
    n, B, H_q, H_kv, cap, T, P = 1, 3, 8, 2, 70, 6, 50
    K, V = cache(n, B, cap, H_kv, 251, dev)
    Kp, Vp = (normal((n, P, H_kv, D), 253 + i, dev) for i in range(2))
    q, qc = normal((n, B, H_q, D), 255, dev), normal((n, B, T, H_q, D), 256, dev)
    far, near = i32([-5, cap + 9, 2 ** 31 - 1], dev), i32([0, cap, cap], dev)
    rows_far, rows = i32([-1, T + 3, 2 ** 31 - 1], dev), i32([0, T, T], dev)

    def accum(lens):
        w = torch.zeros((n, B, 1, cap), device=dev)
        return (*spec.accum_decode_attn(q, K, V, lens, w), w)

    for call in (lambda lens, r, p: spec.window_decode_attn(q, K, V, lens, 30, n_sink=2),
                 lambda lens, r, p: spec.window_attn(qc, K, V, lens, 30, n_sink=2, q_lens=r),
                 lambda lens, r, p: spec.prefix_decode_attn(q, Kp, Vp, K, V, lens, prefix_len=p),
                 lambda lens, r, p: accum(lens)):
        for a, b in zip(call(far, rows_far, i32([P + 4], dev)), call(near, rows, i32([P], dev))):
            assert same_bits(a, b)

    def evict(counts, keep, rows):
        x = bounded(n, B, 1, H_kv, cap, 257, dev)
        kv = normal((2, n, B, T, H_kv, D), 259, dev)
        c = counts.clone()
        spec.evict(*x, c, keep, i32([0, 90, 90], dev), k_new=kv[0], v_new=kv[1], n_new=rows,
                   n_recent=9)
        return (*x, c)

    for a, b in zip(evict(far, i32([cap + 1, -3, cap], dev), rows_far),
                    evict(near, i32([cap, 0, cap], dev), rows)):
        assert same_bits(a, b)


def test_debug_mode_rejects(dev, monkeypatch):
    n, B, H_q, H_kv, cap, T, P = 1, 2, 8, 2, 70, 6, 50
    K, V = cache(n, B, cap, H_kv, 261, dev)
    Kp, Vp = (normal((n, P, H_kv, D), 263 + i, dev) for i in range(2))
    q, qc = normal((n, B, H_q, D), 265, dev), normal((n, B, T, H_q, D), 266, dev)
    ok, bad = i32([70, 0], dev), i32([71, 0], dev)
    w, t = torch.zeros((n, B, 1, cap), device=dev), torch.zeros((n, B, 1, cap), dtype=torch.int32,
                                                                device=dev)
    kv = normal((2, n, B, T, H_kv, D), 267, dev)
    want = spec.window_decode_attn(q, K, V, ok, 30)[0]
    torch.cuda.synchronize()
    monkeypatch.setenv("SPEC_DEBUG", "1")
    assert torch.equal(spec.window_decode_attn(q, K, V, ok, 30)[0], want)
    for call in (lambda: spec.window_decode_attn(q, K, V, bad, 30),
                 lambda: spec.window_attn(qc, K, V, bad, 30),
                 lambda: spec.window_attn(qc, K, V, ok, 30, q_lens=i32([7, 0], dev)),
                 lambda: spec.prefix_decode_attn(q, Kp, Vp, K, V, bad),
                 lambda: spec.prefix_decode_attn(q, Kp, Vp, K, V, ok, prefix_len=i32([51], dev)),
                 lambda: spec.accum_decode_attn(q, K, V, i32([-1, 0], dev), w),
                 lambda: spec.evict(K, V, w, t, bad, ok, ok, k_new=kv[0], v_new=kv[1]),
                 lambda: spec.evict(K, V, w, t, ok, bad, ok, k_new=kv[0], v_new=kv[1]),
                 lambda: spec.evict(K, V, w, t, ok, ok, ok, k_new=kv[0], v_new=kv[1],
                                    n_new=i32([7, 0], dev))):
        with pytest.raises(spec.SpecError) as e:
            call()
        assert e.value.status == 1
    monkeypatch.delenv("SPEC_DEBUG")
    assert not w.any() and ok.tolist() == [70, 0]


@pytest.mark.parametrize("T,cap", [(9, 64), (40, 3000), (300, 300)])
def test_window_in_place(dev, T, cap):
    """The outputs may take the queries' place."""
    K, V = cache(1, 2, cap, 2, 271, dev)
    q = normal((1, 2, T, 8, D), 273, dev)
    lens = i32([cap, cap - 3], dev)
    want, _ = spec.window_attn(q, K, V, lens, 1000, n_sink=1)
    got, _ = spec.window_attn(q, K, V, lens, 1000, n_sink=1, out=q)
    assert got is q and torch.equal(got, want)


@pytest.mark.parametrize("n,B,H_q,H_kv,cap", [(1, 2, 8, 2, 300), (1, 1, 24, 1, 2000),
                                              (16, 8, 32, 8, 130), (1, 3, 6, 3, 20000)])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_decode_odd_values(dev, n, B, H_q, H_kv, cap, odd):
    """The same of the decode entry points: a row of V of the last KV head."""
    counts = [cap - 7 * b for b in range(B)]
    K, V = cache(n, B, cap, H_kv, 281, dev, counts)
    q = normal((n, B, H_q, D), 283, dev)
    l, g, G = n - 1, H_kv - 1, H_q // H_kv
    clean = f64(V[l, 0])
    for t, dim in {counts[0] - 1: 3, 100: 70, 0: 127}.items():
        V[l, 0, t, g, dim] = odd
        clean[t, g, dim] = 0.0
    lens = i32(counts, dev)
    qq, kk = f64(q[l, 0]), f64(K[l, 0])
    L = counts[0]
    want, _, add = dense_oracle.accumulate(qq, kk[:L], clean[:L], 1, SCALE)
    spread, _, _ = dense_oracle.accumulate(qq, kk[:L], np.abs(clean[:L]), 1, SCALE)
    e = weight_error(qq, finite(kk), cap)
    w = torch.zeros((n, B, 1, cap), device=dev)
    p = normal((n, 40, H_kv, D), 285, dev)
    for what, out in (("window", spec.window_decode_attn(q, K, V, lens, cap)[0]),
                      ("accum", spec.accum_decode_attn(q, K, V, lens, w)[0]),
                      ("prefix", spec.prefix_decode_attn(q, p, p, K, V, lens,
                                                         prefix_len=i32([0], dev))[0])):
        got = out[l, 0].double().cpu().numpy()
        heads = slice(g * G, (g + 1) * G)
        for dim in (3, 70, 127):
            at = got[heads, dim]
            assert (np.isnan(at) if odd != odd else at == odd).all(), what
            got[heads, dim] = want[heads, dim]
        check(got, want, 2 * e * spread + 1e-30, what)
    check(w[l, 0, 0, :L].cpu(), add[0], (2 * e + 2.0 ** -19 + H_q * U) * add[0], "weights")
