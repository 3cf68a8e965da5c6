"""Attention over caches that are read in full, and the eviction that keeps
such a cache bounded: what a serving program runs for the layers and phases
that do not select tokens.

* `window_decode_attn`, `window_attn`: a sliding window with a few first tokens
  that stay visible, for one new token per sequence and for chunks of them;
* `prefix_decode_attn`: a batch whose sequences share one long prefix, whose
  rows are read once for all of them;
* `accum_decode_attn`: decode attention that adds each token's weight to a
  running sum, and `evict`, which inserts new rows into a bounded cache in the
  place of those with the least accumulated weight.

`own` chooses between their plain form (elementary torch operations in 32 bits)
and the framework's entry points.  `listed()` names the cases; `draw(rng)`
gives others of the same ranges.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
D = 128   # head dimension


def listed():
    return [
        # One layer of one short chat: launches and latency.
        dict(name="window_decode_b1_l4096", kind="window_decode", layers=1, B=1, L=4096,
             ragged=False, H_q=32, H_kv=8, window=1024, sinks=4),
        # Every layer of an 8B-class model for a batch, a window of 2K.
        dict(name="window_decode_b8_32layers", kind="window_decode", layers=32, B=8, L=8192,
             ragged=False, H_q=32, H_kv=8, window=2048, sinks=4),
        # Prefill of two prompts that the window still covers whole: causal attention.
        dict(name="window_chunk_b2_t4096", kind="window", layers=1, B=2, T=4096, L=4096,
             ragged=False, H_q=32, H_kv=8, window=4096, sinks=4),
        # Prefill of a prompt far longer than the window.
        dict(name="window_chunk_t8192_w1024", kind="window", layers=1, B=1, T=8192, L=8192,
             ragged=False, H_q=32, H_kv=8, window=1024, sinks=16),
        # A ragged batch of chunks, seven query heads per KV head, odd sizes, padding.
        dict(name="window_chunk_b5_t257_g7", kind="window", layers=1, B=5, T=257, L=3001,
             ragged=True, H_q=28, H_kv=4, window=777, sinks=3),
        # A few answers sampled from one short prompt.
        dict(name="prefix_b4_p1000", kind="prefix", layers=1, B=4, P=1000, L=128, ragged=False,
             H_q=32, H_kv=8),
        # A small batch on a long document, odd lengths.
        dict(name="prefix_b16_p20011", kind="prefix", layers=2, B=16, P=20011, L=777,
             ragged=True, H_q=32, H_kv=8),
        # A large batch on a long shared context.
        dict(name="prefix_b64_p32768_4layers", kind="prefix", layers=4, B=64, P=32768, L=1024,
             ragged=True, H_q=32, H_kv=8),
        # One layer of a small ragged batch, the weights summed over all heads.
        dict(name="accum_b3_l1500_g8", kind="accum", layers=1, B=3, L=1500, ragged=True, H_q=64,
             H_kv=8, per_head=False),
        # Every layer of a model over caches bounded at 2K, weights per KV head.
        dict(name="accum_b8_l2048_32layers", kind="accum", layers=32, B=8, L=2048, ragged=False,
             H_q=32, H_kv=8, per_head=True),
        # One decode step's insertion into the bounded caches of every layer.
        dict(name="evict_b8_k2048_32layers", kind="evict", layers=32, B=8, keep=2048, new=1,
             full=True, H_kv=8, per_head=True, recent=256, sinks=4),
        # A block of new tokens per sequence into long caches, whole tokens at a time.
        dict(name="evict_b4_k8192_m512", kind="evict", layers=8, B=4, keep=8192, new=512,
             full=True, H_kv=8, per_head=False, recent=1024, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window_decode", "window", "window", "prefix", "prefix", "accum", "evict"])
    H_kv = rng.choice([1, 2, 4, 8])
    H_q = H_kv * rng.choice([1, 3, 4, 7, 8, 16])
    ragged = rng.random() < 0.5
    c = dict(kind=kind, layers=_log(rng, 1, 32), B=_log(rng, 1, 32))
    if kind == "window_decode":
        c.update(L=_log(rng, 1, 32768), ragged=ragged, H_q=H_q, H_kv=H_kv,
                 window=_log(rng, 16, 4096), sinks=rng.choice([0, 1, 4, 16]))
        return _fit(c, lambda c: c["layers"] * c["B"] * c["L"] * H_kv, 1 << 23)
    if kind == "window":
        c.update(layers=1, B=_log(rng, 1, 8), T=_log(rng, 2, 8192), ragged=ragged, H_q=H_q,
                 H_kv=H_kv, sinks=rng.choice([0, 1, 4, 16]))
        c["L"] = c["T"] + rng.choice([0, _log(rng, 1, 8192)])
        c["window"] = rng.choice([c["L"], _log(rng, 16, 4096)])
        c = _fit(c, lambda c: c["B"] * c["T"] * c["L"] * H_q, 1 << 30, ("B", "T"))
        c["L"] = max(c["L"], c["T"])
        return c
    if kind == "prefix":
        c.update(layers=_log(rng, 1, 4), B=_log(rng, 2, 128), P=_log(rng, 64, 65536),
                 L=_log(rng, 1, 2048), ragged=ragged, H_q=H_q, H_kv=H_kv)
        return _fit(c, lambda c: c["layers"] * c["B"] * (H_q * c["P"] + 16 * H_kv * c["L"]),
                    1 << 28)
    if kind == "accum":
        c.update(L=_log(rng, 16, 32768), ragged=ragged, H_q=H_q, H_kv=H_kv,
                 per_head=rng.random() < 0.5)
        return _fit(c, lambda c: c["layers"] * c["B"] * c["L"] * max(H_kv, H_q // 4), 1 << 22)
    c.update(keep=_log(rng, 64, 16384), full=rng.random() < 0.7, H_kv=H_kv,
             per_head=rng.random() < 0.5, sinks=rng.choice([0, 1, 4, 16]))
    c["new"] = _log(rng, 1, max(1, c["keep"] // 8))
    c["recent"] = max(c["new"], c["keep"] // rng.choice([4, 8, 16]))
    return _fit(c, lambda c: c["layers"] * c["B"] * c["keep"] * H_kv, 1 << 22)


def _fit(c, cost, most, shrink=("layers", "B")):
    """A drawn case costs no more than the largest listed ones."""
    while cost(c) > most:
        name = max(shrink, key=lambda s: c[s])
        if c[name] == 1:
            c["P" if "P" in c else "keep" if "keep" in c else "L"] //= 2
        else:
            c[name] //= 2
    return c


# ------------------------------------------------------------------ inputs

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFF)
    return g


def _normal(shape, seed, salt):
    t = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    g = _gen(seed, salt)
    for part in t:
        part.normal_(generator=g)
    return t


def _ints(lo, hi, B, ragged, seed, salt):
    """One length per sequence: hi, or somewhere in [lo, hi]."""
    if not ragged:
        return torch.full((B,), hi, dtype=torch.int32, device=DEV)
    return torch.randint(lo, hi + 1, (B,), generator=_gen(seed, salt), device=DEV).to(torch.int32)


def _inputs(c, seed):
    kind, n, B, H_kv = c["kind"], c["layers"], c["B"], c["H_kv"]
    if kind == "evict":
        cap, m = c["keep"], c["new"]
        sets = H_kv if c["per_head"] else 1
        x = dict(K=_normal((n, B, cap, H_kv, D), seed, 1), V=_normal((n, B, cap, H_kv, D), seed, 2),
                 k_new=_normal((n, B, m, H_kv, D), seed, 3),
                 v_new=_normal((n, B, m, H_kv, D), seed, 4))
        x["counts"] = _ints(0, cap, B, not c["full"], seed, 5)
        x["keep"] = torch.full((B,), cap, dtype=torch.int32, device=DEV)
        # Accumulated weights have a heavy tail.  The tokens seen so far number
        # several times the cache, and stand in its slots in no order.
        u = torch.rand((n, B, sets, cap), generator=_gen(seed, 6), device=DEV)
        x["weights"] = (0.01 / (u + 1e-3)).contiguous()
        order = torch.rand((n, B, sets, cap), generator=_gen(seed, 7), device=DEV).argsort(-1)
        x["tokens"] = (order * 4 + 3).to(torch.int32).contiguous()
        x["pos"] = torch.full((B,), 4 * cap, dtype=torch.int32, device=DEV)
        return x
    H_q, L = c["H_q"], c["L"]
    x = dict(K=_normal((n, B, L, H_kv, D), seed, 1), V=_normal((n, B, L, H_kv, D), seed, 2))
    if kind == "window":
        x["q"] = _normal((n, B, c["T"], H_q, D), seed, 3)
        x["q_lens"] = _ints(0, c["T"], B, c["ragged"], seed, 4)
        more = _ints(0, L - c["T"], B, c["ragged"], seed, 5)
        x["lens"] = x["q_lens"] + more
        return x
    x["q"] = _normal((n, B, H_q, D), seed, 3)
    x["lens"] = _ints(0, L, B, c["ragged"], seed, 4)
    if kind == "prefix":
        x["K_prefix"] = _normal((n, c["P"], H_kv, D), seed, 6)
        x["V_prefix"] = _normal((n, c["P"], H_kv, D), seed, 7)
    elif kind == "accum":
        sets = H_kv if c["per_head"] else 1
        x["weights"] = torch.rand((n, B, sets, L), generator=_gen(seed, 8), device=DEV)
    return x


def prepare(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    x["case"] = c
    if "q" in x:   # a serving program keeps its outputs
        kind = torch.bfloat16 if c["kind"] == "window" else torch.float32
        x["out"] = torch.zeros(x["q"].shape, dtype=kind, device=DEV)
        x["lse"] = torch.zeros(x["q"].shape[:-1], dtype=torch.float32, device=DEV)
    return x


# ------------------------------------------------------------------ the plain forms

def _grouped(t, H_kv):
    """[n][B][rows][H_q][D] -> [n][B][H_kv][G rows][D] in 32 bits, heads outermost."""
    n, B, T, H, _ = t.shape
    t = t.view(n, B, T, H_kv, H // H_kv, D).permute(0, 1, 3, 4, 2, 5).float()
    return t.reshape(n, B, H_kv, H // H_kv * T, D)


def _rows(t):
    """[n][B][L][H_kv][D] -> [n][B][H_kv][L][D] in 32 bits."""
    return t.permute(0, 1, 3, 2, 4).float().contiguous()


def _softmax_parts(s):
    """exp(s - max), its sum and log-sum-exp over the last axis; a row of nothing
    but -inf has sum 0 and -inf."""
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = e.sum(-1, keepdim=True)
    return e, z, (m + torch.log(z)).squeeze(-1)


def _attend(q, k, v, seen):
    """q [n][B][H_kv][R][D], k and v [n][B][H_kv][L][D], seen broadcast over
    [n][B][H_kv][R][L]: outputs, log-sum-exps, weights."""
    s = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    s = s.masked_fill_(~seen, -math.inf)
    e, z, lse = _softmax_parts(s)
    p = e / torch.where(z == 0, torch.ones_like(z), z)
    return torch.matmul(p, v), lse, p


def _plain_window_decode(x, c):
    """The visible rows are gathered, so that the cache behind the window is not read."""
    n, B, H_q, _ = x["q"].shape
    H_kv, L, W, S = c["H_kv"], c["L"], c["window"], c["sinks"]
    lens = x["lens"].long()[:, None]
    j = torch.arange(min(L, W + S), device=DEV)[None, :]
    t = torch.where(j < S, j, j + torch.clamp(lens - W - S, min=0))       # [B][rows]
    seen = t < lens
    t = torch.where(seen, t, torch.zeros_like(t))
    at = t[None, :, :, None, None].expand(n, B, t.shape[1], H_kv, D)
    k, v = _rows(torch.gather(x["K"], 2, at)), _rows(torch.gather(x["V"], 2, at))
    out, lse, _ = _attend(_grouped(x["q"][:, :, None], H_kv), k, v, seen[None, :, None, None, :])
    return dict(out=out.reshape(n, B, H_q, D), lse=lse.reshape(n, B, H_q))


def _plain_window(x, c):
    n, B, T, H_q, _ = x["q"].shape
    H_kv, L, G = c["H_kv"], c["L"], H_q // c["H_kv"]
    lens, rows = x["lens"].long()[:, None, None], x["q_lens"].long()[:, None, None]
    i, t = torch.arange(T, device=DEV)[None, :, None], torch.arange(L, device=DEV)[None, None, :]
    p = lens - rows + i
    seen = (t <= p) & ((t < c["sinks"]) | (t > p - c["window"]))           # [B][T][L]
    seen = seen.repeat(1, G, 1)[None, :, None]
    out, lse, _ = _attend(_grouped(x["q"], H_kv), _rows(x["K"]), _rows(x["V"]), seen)
    out = out.view(n, B, H_kv, G, T, D).permute(0, 1, 4, 2, 3, 5).reshape(n, B, T, H_q, D)
    lse = lse.view(n, B, H_kv, G, T).permute(0, 1, 4, 2, 3).reshape(n, B, T, H_q)
    # queries behind a sequence's last one are left as they were
    here = (torch.arange(T, device=DEV)[None, :] < x["q_lens"][:, None])[None, :, :, None]
    return dict(out=torch.where(here[..., None], out, torch.zeros_like(out)).to(torch.bfloat16),
                lse=torch.where(here, lse, torch.zeros_like(lse)))


def _plain_prefix(x, c):
    """The prefix once for every sequence, the own tokens per sequence, and the
    two softmaxes joined."""
    n, B, H_q, _ = x["q"].shape
    H_kv, L, G = c["H_kv"], c["L"], H_q // c["H_kv"]
    q = x["q"].float().view(n, B, H_kv, G, D)
    qp = q.permute(0, 2, 1, 3, 4).reshape(n, H_kv, B * G, D)
    kp, vp = x["K_prefix"].float().transpose(1, 2), x["V_prefix"].float().transpose(1, 2)
    scale = 1.0 / math.sqrt(D)
    s0 = (torch.matmul(qp, kp.transpose(-1, -2)) * scale).view(n, H_kv, B, G, -1)
    s0 = s0.transpose(1, 2)                                                # [n][B][H_kv][G][P]
    s1 = torch.matmul(q, _rows(x["K"]).transpose(-1, -2)) * scale          # [n][B][H_kv][G][L]
    seen = torch.arange(L, device=DEV)[None, :] < x["lens"][:, None]
    s1 = s1.masked_fill_(~seen[None, :, None, None, :], -math.inf)
    m = torch.maximum(s0.amax(-1, keepdim=True), s1.amax(-1, keepdim=True))
    e0, e1 = torch.exp(s0 - m), torch.exp(s1 - m)
    z = e0.sum(-1, keepdim=True) + e1.sum(-1, keepdim=True)
    o0 = torch.matmul(e0.transpose(1, 2).reshape(n, H_kv, B * G, -1), vp)
    o0 = o0.view(n, H_kv, B, G, D).transpose(1, 2)
    out = (o0 + torch.matmul(e1, _rows(x["V"]))) / z
    return dict(out=out.reshape(n, B, H_q, D), lse=(m + torch.log(z)).reshape(n, B, H_q))


def _plain_accum(x, c):
    n, B, H_q, _ = x["q"].shape
    seen = torch.arange(c["L"], device=DEV)[None, :] < x["lens"][:, None]
    out, lse, p = _attend(_grouped(x["q"][:, :, None], c["H_kv"]), _rows(x["K"]), _rows(x["V"]),
                          seen[None, :, None, None, :])
    p = p.sum(3)                                                           # [n][B][H_kv][L]
    x["weights"] += p if c["per_head"] else p.sum(2, keepdim=True)
    return dict(out=out.reshape(n, B, H_q, D), lse=lse.reshape(n, B, H_q), weights=x["weights"])


def _plain_evict(x, c):
    """Here the cache's capacity is its budget, so that only new rows move: each
    into a slot that holds nothing or whose row is evicted."""
    n, B, S, cap = x["weights"].shape
    H_kv, m = c["H_kv"], c["new"]
    count, pos = x["counts"].long()[:, None, None], x["pos"].long()[:, None, None]
    after = torch.minimum(x["keep"].long()[:, None, None], count + m)
    slot = torch.arange(cap, device=DEV)
    held = slot < count
    safe = (x["tokens"] >= pos + m - c["recent"]) | (x["tokens"] < c["sinks"])
    w = torch.where(torch.isnan(x["weights"]), torch.full_like(x["weights"], -math.inf),
                    x["weights"])
    w = torch.where(safe, torch.full_like(w, math.inf), w)
    w = torch.where(held, w, torch.full_like(w, -math.inf))
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    rank = torch.zeros_like(order).scatter_(-1, order, slot.expand_as(order))
    kept = held & (rank < after - m)
    free = (slot < after) & ~kept
    # the first m slots of `free`, ascending
    at = torch.sort(free.to(torch.int8), dim=-1, descending=True, stable=True).indices[..., :m]
    x["weights"].scatter_(-1, at, 0.0)
    x["tokens"].scatter_(-1, at, (pos + torch.arange(m, device=DEV)).to(torch.int32)
                         .expand(n, B, S, m))
    at = at.transpose(-1, -2)[..., None].expand(n, B, m, S, H_kv // S * D)  # [n][B][m][S][..]
    x["K"].view(n, B, cap, S, -1).scatter_(2, at, x["k_new"].view(n, B, m, S, -1))
    x["V"].view(n, B, cap, S, -1).scatter_(2, at, x["v_new"].view(n, B, m, S, -1))
    x["counts"].copy_(after[:, 0, 0])


# ------------------------------------------------------------------ one pass

def _own(x, c):
    """The framework's calls, with a workspace that a program keeps."""
    import paper_2512_00722_amd as spec

    kind, n, B, H_kv = c["kind"], c["layers"], c["B"], c["H_kv"]
    if "ws" not in x:
        op = dict(window_decode=spec.DENSE_WINDOW_DECODE, window=spec.DENSE_WINDOW,
                  prefix=spec.DENSE_PREFIX_DECODE, accum=spec.DENSE_ACCUM_DECODE,
                  evict=spec.DENSE_EVICT)[kind]
        dims = spec.DenseDims.make(B=B, L_cap=x["K"].shape[2], n_layers=n,
                                   H_q=c.get("H_q", H_kv), H_kv=H_kv,
                                   T=c["T"] if kind == "window" else c.get("new", 1),
                                   window=c.get("window", 0), n_sink=c.get("sinks", 0),
                                   P_cap=c.get("P", 0), n_sets=H_kv if c.get("per_head") else 1,
                                   n_recent=c.get("recent", 0))
        x["ws"] = torch.empty(max(16, spec.dense_workspace_size(dims, op)), dtype=torch.uint8,
                              device=DEV)
    ws = x["ws"]
    if kind == "window_decode":
        out, lse = spec.window_decode_attn(x["q"], x["K"], x["V"], x["lens"], c["window"],
                                           n_sink=c["sinks"], out=x["out"], lse=x["lse"], ws=ws)
    elif kind == "window":
        out, lse = spec.window_attn(x["q"], x["K"], x["V"], x["lens"], c["window"],
                                    n_sink=c["sinks"], q_lens=x["q_lens"], out=x["out"],
                                    lse=x["lse"], ws=ws)
    elif kind == "prefix":
        out, lse = spec.prefix_decode_attn(x["q"], x["K_prefix"], x["V_prefix"], x["K"], x["V"],
                                           x["lens"], out=x["out"], lse=x["lse"], ws=ws)
    elif kind == "accum":
        out, lse = spec.accum_decode_attn(x["q"], x["K"], x["V"], x["lens"], x["weights"],
                                          out=x["out"], lse=x["lse"], ws=ws)
        return dict(out=out, lse=lse, weights=x["weights"])
    else:
        spec.evict(x["K"], x["V"], x["weights"], x["tokens"], x["counts"], x["keep"], x["pos"],
                   k_new=x["k_new"], v_new=x["v_new"], n_recent=c["recent"], n_sink=c["sinks"],
                   ws=ws)
        return None
    return dict(out=out, lse=lse)


def run(x):
    c = x["case"]
    if own:
        r = _own(x, c)
    else:
        r = dict(window_decode=_plain_window_decode, window=_plain_window, prefix=_plain_prefix,
                 accum=_plain_accum, evict=_plain_evict)[c["kind"]](x, c)
    if c["kind"] != "evict":
        return r
    # the next insertion's tokens follow these
    x["pos"] += c["new"]
    return dict(K=x["K"], V=x["V"], weights=x["weights"], tokens=x["tokens"], counts=x["counts"])


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = dict(case)
    kind, n, B, H_kv = c["kind"], c["layers"], c["B"], c["H_kv"]
    half = 0.5 if c.get("ragged") else 1.0       # expected share of the longest length
    row = H_kv * D * 2 * 2                       # K and V of a token
    if kind == "evict":
        # weights and tokens of every slot; the new rows, read and written
        sets = H_kv if c["per_head"] else 1
        slots = n * B * sets * c["keep"] * (1.0 if c["full"] else 0.5)
        return dict(bytes=slots * 8 + 2 * n * B * c["new"] * row, flops=slots)
    H_q = c["H_q"]
    io = n * B * H_q * (D * 6 + 4)               # queries, outputs, log-sum-exps
    if kind == "window_decode":
        toks = n * B * min(c["L"] * half, c["window"] + c["sinks"])
        return dict(bytes=toks * row + io, flops=4.0 * toks * H_q * D)
    if kind == "window":
        T, L, W = c["T"] * half, c["T"] * half + (c["L"] - c["T"]) * half, c["window"] + c["sinks"]
        # pairs: the causal triangle's last T rows, cut to W visible tokens
        full = max(0.0, min(T, L - W))           # rows that see W tokens
        rest = T - full                          # rows that see all before them
        low = L - T + 1
        pairs = B * (full * W + rest * (low + min(L, max(W, low))) / 2)
        read = B * min(L, T + W)
        return dict(bytes=read * row + B * T * H_q * (D * 4 + 4), flops=4.0 * pairs * H_q * D)
    if kind == "prefix":
        own_toks = n * B * c["L"] * half
        return dict(bytes=(n * c["P"] + own_toks) * row + io,
                    flops=4.0 * (n * B * c["P"] + own_toks) * H_q * D)
    toks = n * B * c["L"] * half
    sets = H_kv if c["per_head"] else 1
    return dict(bytes=toks * (row + 8 * sets) + io, flops=4.0 * toks * H_q * D)


# ------------------------------------------------------------------ in 64 bits

def _exact_rows(q, k, v, seen):
    """q [R][D], k and v [L][D] of one KV head, seen [R][L]: outputs, lse, weights."""
    s = q.double() @ k.double().t().contiguous() / math.sqrt(D)
    s[~seen] = -math.inf
    lse = torch.logsumexp(s, dim=-1)
    p = torch.nan_to_num(torch.softmax(s, dim=-1), nan=0.0)
    return p @ v.double(), lse, p


def _exact_evict(x, c):
    """Slot by slot from the definition, on the host's indices."""
    n, B, S, cap = x["weights"].shape
    m, per = c["new"], c["H_kv"] // S
    w_all, t_all = x["weights"].cpu().numpy(), x["tokens"].cpu().numpy()
    counts, pos = x["counts"].tolist(), x["pos"].tolist()
    weights, tokens = x["weights"].double(), x["tokens"].clone()
    K, V = x["K"].clone(), x["V"].clone()
    for l in range(n):
        for b in range(B):
            held = counts[b]
            after = min(cap, held + m)
            keep = after - m
            for s in range(S):
                w, t = w_all[l, b, s, :held], t_all[l, b, s, :held]
                safe = (t >= pos[b] + m - c["recent"]) | (t < c["sinks"])
                first = np.lexsort((np.arange(held), np.where(safe, 0.0, -w), ~safe))
                stay = np.zeros(after, dtype=bool)
                stay[first[:keep]] = True
                free = torch.from_numpy(np.nonzero(~stay)[0]).to(DEV)
                heads = slice(s * per, (s + 1) * per)
                K[l, b, free, heads] = x["k_new"][l, b, :, heads]
                V[l, b, free, heads] = x["v_new"][l, b, :, heads]
                weights[l, b, s, free] = 0.0
                tokens[l, b, s, free] = pos[b] + torch.arange(m, dtype=torch.int32, device=DEV)
    after = torch.tensor([min(cap, h + m) for h in counts], dtype=torch.int32, device=DEV)
    return dict(K=K, V=V, weights=weights, tokens=tokens, counts=after)


def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    kind, n, B, H_kv = c["kind"], c["layers"], c["B"], c["H_kv"]
    if kind == "evict":
        return _exact_evict(x, c) if n * B * c["keep"] * (H_kv if c["per_head"] else 1) \
            <= 1 << 23 else None
    q, K, V = x["q"], x["K"], x["V"]
    lens = x["lens"].tolist()
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(q.shape[:-1], dtype=torch.float64, device=DEV)
    weights = x["weights"].double() if kind == "accum" else None
    G = c["H_q"] // H_kv
    for l in range(n):
        for g in range(H_kv):
            hs = slice(g * G, (g + 1) * G)
            if kind == "prefix":
                kp, vp = x["K_prefix"][l, :, g].double(), x["V_prefix"][l, :, g].double()
            for b in range(B):
                L = lens[b]
                if kind == "window":
                    rows = int(x["q_lens"][b])
                    if rows == 0:
                        continue
                    p = torch.arange(L - rows, L, device=DEV)[:, None]
                    t = torch.arange(L, device=DEV)[None, :]
                    seen = (t <= p) & ((t < c["sinks"]) | (p - t < c["window"]))
                    for h in range(g * G, (g + 1) * G):
                        o, z, _ = _exact_rows(q[l, b, :rows, h], K[l, b, :L, g], V[l, b, :L, g],
                                              seen)
                        out[l, b, :rows, h], lse[l, b, :rows, h] = o, z
                    continue
                if kind == "window_decode":
                    lo = max(0, L - c["window"])
                    t = torch.cat([torch.arange(min(c["sinks"], lo), device=DEV),
                                   torch.arange(lo, L, device=DEV)])
                    k, v = K[l, b, t, g], V[l, b, t, g]
                else:
                    k, v = K[l, b, :L, g], V[l, b, :L, g]
                if kind == "prefix":
                    k, v = torch.cat([kp, k.double()]), torch.cat([vp, v.double()])
                if k.shape[0] == 0:
                    lse[l, b, hs] = -math.inf
                    continue
                o, z, p = _exact_rows(q[l, b, hs], k, v, torch.ones(
                    (G, k.shape[0]), dtype=torch.bool, device=DEV))
                out[l, b, hs], lse[l, b, hs] = o, z
                if kind == "accum":
                    weights[l, b, g if c["per_head"] else 0, :L] += p.sum(0)
    if kind == "accum":
        return dict(out=out, lse=lse, weights=weights)
    return dict(out=out, lse=lse)
