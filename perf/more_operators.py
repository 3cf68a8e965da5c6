"""KV caches held in 4 or 8 bits: what a serving program runs whose caches do not
fit, or whose decode steps are bound by the bytes of their caches.

A cache's rows are held in groups of 32 along the head dimension: elements of 4
bits (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives) or of 8 bits (e4m3), times a
power of two per group, the least with which no element errs by more than half a
step (2^X with the largest magnitude at most 7 2^X, or 448 2^X).

* `quant_append` quantises new tokens' rows as they are written, `quant_read`
  gives rows back;
* `quant_decode_attn`: decode attention over all rows or a sliding window with
  sinks;
* `quant_sparse_decode_attn`: decode attention over selected rows.

`own` chooses between their plain form (elementary torch operations in 32 bits)
and the framework's entry points.  `listed()` names the cases; `draw(rng)`
gives others of the same ranges.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
D = 128      # head dimension
GROUP = 32   # elements of a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
NAN_SCALE = 255


def listed():
    return [
        # One decode step's new token in every layer, and its rows as the caches hold them:
        # launches and latency.
        dict(name="append_b1_t1_32layers", kind="append", layers=32, B=1, T=1, L=4096,
             ragged=False, H_kv=8, bits=4),
        # A ragged batch of chunks, odd sizes, 8 bits.
        dict(name="append_b5_t257_8bit", kind="append", layers=8, B=5, T=257, L=3001, ragged=True,
             H_kv=4, bits=8),
        # Prefill: two prompts' rows of some layers, written and read back for the chunk's
        # own attention, which so sees the values that decoding will see.
        dict(name="append_b2_t8192_8layers", kind="append", layers=8, B=2, T=8192, L=8192,
             ragged=False, H_kv=8, bits=4),
        # One long cache read in full, before attention of a chunk over it; odd lengths.
        dict(name="read_b2_l20011_8bit", kind="read", layers=4, B=2, L=20011, k=0, ragged=True,
             H_kv=8, sets=1, bits=8),
        # The selected rows of a batch in compact form.
        dict(name="read_b8_k2048_8layers", kind="read", layers=8, B=8, L=32768, k=2048,
             ragged=False, H_kv=8, sets=1, bits=4),
        # One layer of one short chat: launches and latency.
        dict(name="decode_b1_l4096", kind="decode", layers=1, B=1, L=4096, ragged=False, H_q=32,
             H_kv=8, window=0, sinks=0, bits=4),
        # Every layer of an 8B-class model for a batch of long contexts.
        dict(name="decode_b8_l32768_32layers", kind="decode", layers=32, B=8, L=32768,
             ragged=False, H_q=32, H_kv=8, window=0, sinks=0, bits=4),
        # The same caches in 8 bits, a window of 2K for a larger batch.
        dict(name="decode_b32_w2048_8bit", kind="decode", layers=16, B=32, L=8192, ragged=False,
             H_q=32, H_kv=8, window=2048, sinks=4, bits=8),
        # A ragged batch of odd lengths, seven query heads per KV head.
        dict(name="decode_b5_l20011_g7", kind="decode", layers=4, B=5, L=20011, ragged=True,
             H_q=28, H_kv=4, window=0, sinks=0, bits=4),
        # One sequence's selection in one layer: latency.
        dict(name="sparse_b1_l4096_k512", kind="sparse", layers=1, B=1, L=4096, k=512,
             ragged=False, H_q=32, H_kv=8, sets=1, bits=4),
        # The selection of a decode step in every layer of a batch of long contexts.
        dict(name="sparse_b8_l32768_k2048", kind="sparse", layers=32, B=8, L=32768, k=2048,
             ragged=False, H_q=32, H_kv=8, sets=1, bits=4),
        # One set of tokens per KV head, eight query heads each, 8 bits, ragged.
        dict(name="sparse_heads_k4096_8bit", kind="sparse", layers=8, B=3, L=65536, k=4096,
             ragged=True, H_q=64, H_kv=8, sets=8, bits=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "read", "decode", "decode", "sparse", "sparse"])
    H_kv = rng.choice([1, 2, 4, 8])
    c = dict(kind=kind, layers=_log(rng, 1, 32), B=_log(rng, 1, 32), H_kv=H_kv,
             ragged=rng.random() < 0.5, bits=rng.choice([4, 8]))
    if kind == "append":
        c["T"] = _log(rng, 1, 8192)
        c["L"] = c["T"] + rng.choice([0, _log(rng, 1, 4096)])
        c = _fit(c, lambda c: c["layers"] * c["B"] * c["L"] * H_kv, 1 << 20)
        c["T"] = min(c["T"], c["L"])
        return c
    c["L"] = _log(rng, 1, 65536)
    if kind == "decode":
        c.update(H_q=H_kv * rng.choice([1, 3, 4, 7, 8, 16]),
                 window=rng.choice([0, 0, _log(rng, 16, 4096)]), sinks=rng.choice([0, 1, 4, 16]))
        return _fit(c, lambda c: c["layers"] * c["B"] * c["L"] * c["H_q"], 1 << 26)
    c["sets"] = rng.choice([1, 1, H_kv])
    c["k"] = _log(rng, 1, 4096)
    if kind == "read" and rng.random() < 0.3:
        c.update(k=0, sets=1)
    if kind == "sparse":
        c["H_q"] = H_kv * rng.choice([1, 3, 4, 7, 8, 16])
    # the caches behind a selection, and the rows selected
    c = _fit(c, lambda c: c["layers"] * c["B"] * c["L"] * H_kv, 1 << 24)
    c = _fit(c, lambda c: c["layers"] * c["B"] * (c["k"] or c["L"]) * c.get("H_q", 2 * H_kv),
             1 << 21)
    c["k"] = min(c["k"], c["L"])
    return c


def _fit(c, cost, most, shrink=("layers", "B")):
    """A drawn case costs no more than the largest listed ones."""
    while cost(c) > most:
        name = max(shrink, key=lambda s: c[s])
        if c[name] == 1:
            c["k" if c.get("k", 0) > 1 and cost(dict(c, L=1)) > most else "L"] //= 2
        else:
            c[name] //= 2
    return c


# ------------------------------------------------------------------ the plain forms: held values

def _tables():
    """Values of 4-bit elements, and of scales' bytes."""
    grid = torch.tensor(GRID, device=DEV)
    scale = torch.ldexp(torch.ones(256, device=DEV), torch.arange(256, device=DEV) - 127)
    scale[NAN_SCALE] = math.nan
    return torch.cat([grid, -grid]), scale


def _quantise(x, bits):
    """x [.., D] bf16 -> elements uint8 [.., D * bits / 8], scales uint8 [.., D / GROUP]."""
    g = x.float().unflatten(-1, (D // GROUP, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(g).all(-1, keepdim=True)
    m, e = torch.frexp(torch.where(bad, torch.ones_like(top), top))   # top = m 2^e, .5 <= m < 1
    X = e - (3 if bits == 4 else 9) + (m > 0.875).to(e.dtype)
    X = torch.where(top == 0, torch.full_like(X, -111), X)
    X = X.clamp(-111, 125 if bits == 4 else 119)
    y = torch.ldexp(torch.where(bad, torch.zeros_like(g), g), -X)
    sign = torch.signbit(y)
    if bits == 4:
        a = y.abs()
        # borders halfway between the grid's values; one at a border goes to the even element
        code = (a > 0.25).to(torch.uint8)
        code += a >= 0.75
        code += a > 1.25
        code += a >= 1.75
        code += a > 2.5
        code += a >= 3.5
        code += a > 5.0
        code = (code + 8 * sign.to(torch.uint8)).flatten(-2)
        code = code[..., 0::2] + 16 * code[..., 1::2]
    else:
        code = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    scale = torch.where(bad, torch.full_like(X, NAN_SCALE - 127), X) + 127
    return code, scale.to(torch.uint8).squeeze(-1)


def _values(code, scale, bits, tables):
    """Elements [.., D * bits / 8] and scales [.., D / GROUP] -> their values [.., D] in 32 bits."""
    grid, powers = tables
    if bits == 4:
        v = torch.stack([grid[(code & 15).long()], grid[(code >> 4).long()]], -1).flatten(-2)
    else:
        v = code.view(torch.float8_e4m3fn).float()
    v = v.unflatten(-1, (D // GROUP, GROUP)) * powers[scale.long()][..., None]
    return v.flatten(-2)


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


def _cache(c, seed, filled=True):
    """A cache's elements and scales; filled: of normal rows, some channels of K
    larger than the others."""
    n, B, L, H_kv, bits = c["layers"], c["B"], c["L"], c["H_kv"], c["bits"]
    k, v = (torch.zeros((n, B, L, H_kv, D * bits // 8), dtype=torch.uint8, device=DEV)
            for _ in range(2))
    s = torch.zeros((n, B, L, H_kv, 2, D // GROUP), dtype=torch.uint8, device=DEV)
    if filled:
        g = _gen(seed, 1)
        part = max(1, (1 << 25) // (L * H_kv * D))    # sequences at a time
        for l in range(n):
            for b in range(0, B, part):
                x = torch.empty((min(part, B - b), L, H_kv, D), dtype=torch.bfloat16, device=DEV)
                x.normal_(generator=g)
                x[..., ::19] *= 4
                k[l, b:b + part], s[l, b:b + part, :, :, 0] = _quantise(x, bits)
                x.normal_(generator=g)
                v[l, b:b + part], s[l, b:b + part, :, :, 1] = _quantise(x, bits)
    return k, v, s


def _selection(c, counts, seed):
    """Ascending distinct tokens, counts[b] of them, then -1: [B][sets][k]."""
    B, L, k = c["B"], c["L"], c["k"]
    idx = torch.full((B, c["sets"], k), -1, dtype=torch.int32, device=DEV)
    g = _gen(seed, 5)
    for b, n in enumerate(counts.tolist()):
        order = torch.rand((c["sets"], L), generator=g, device=DEV).argsort(-1)[:, :n]
        idx[b, :, :n] = order.sort(-1).values.to(torch.int32)
    return idx if c["sets"] > 1 else idx[:, 0].contiguous()


def _inputs(c, seed):
    kind, n, B, H_kv, L = c["kind"], c["layers"], c["B"], c["H_kv"], c["L"]
    x = {}
    if kind == "append":
        T = c["T"]
        x["k_new"], x["v_new"] = (_normal((n, B, T, H_kv, D), seed, s) for s in (2, 3))
        x["k_new"][..., ::19] *= 4
        x["n_new"] = _ints(0, T, B, c["ragged"], seed, 4)
        x["pos"] = _ints(0, L - T, B, True, seed, 6)
        x["idx"] = x["pos"][:, None] + torch.arange(T, dtype=torch.int32, device=DEV)
        return x
    if kind == "decode":
        x["lens"] = _ints(0, L, B, c["ragged"], seed, 4)
    elif c["k"]:
        x["counts"] = _ints(0, c["k"], B, c["ragged"], seed, 4)
        x["idx"] = _selection(c, x["counts"], seed)
    else:
        x["counts"] = _ints(0, L, B, c["ragged"], seed, 4)
    if "H_q" in c:
        x["q"] = _normal((n, B, c["H_q"], D), seed, 2)
    return x


def prepare(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    x["case"] = c
    x["cache"] = _cache(c, seed, filled=c["kind"] != "append")
    # a serving program keeps its outputs
    if "q" in x:
        x["out"] = torch.zeros(x["q"].shape, dtype=torch.float32, device=DEV)
        x["lse"] = torch.zeros(x["q"].shape[:-1], dtype=torch.float32, device=DEV)
    else:
        rows = c["T"] if c["kind"] == "append" else c["k"] or c["L"]
        x["rows"] = tuple(torch.zeros((c["layers"], c["B"], rows, c["H_kv"], D),
                                      dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return x


# ------------------------------------------------------------------ the plain forms: passes

def _plain_append(x, c):
    """The rows that there are, at their places: rows behind a sequence's last are not
    written."""
    k, v, s = x["cache"]
    T = c["T"]
    here = torch.arange(T, device=DEV)[None, :] < x["n_new"][:, None]
    b, i = here.nonzero(as_tuple=True)
    t = x["idx"].long()[b, i]
    for j, (new, code) in enumerate(((x["k_new"], k), (x["v_new"], v))):
        held, scale = _quantise(new[:, b, i], c["bits"])
        code[:, b, t] = held
        s[:, b, t, :, j] = scale
    out = []
    tables = _tables()
    for j, code in enumerate((k, v)):
        rows = torch.zeros_like(x["rows"][0])
        rows[:, b, i] = _values(code[:, b, t], s[:, b, t, :, j], c["bits"],
                                tables).to(torch.bfloat16)
        out.append(rows)
    return dict(K=out[0], V=out[1])


def _picked(x, c, layer):
    """A layer's rows [B][k][H_kv] that a selection names (padding: row 0): elements of
    K and V, scales."""
    idx = x["idx"].clamp(min=0).long()
    if idx.dim() == 2:
        idx = idx[:, None]
    idx = idx.expand(-1, c["H_kv"], -1).transpose(1, 2)                     # [B][k][H_kv]
    b = torch.arange(c["B"], device=DEV)[:, None, None]
    h = torch.arange(c["H_kv"], device=DEV)[None, None, :]
    return [t[layer][b, idx, h] for t in x["cache"]]


def _plain_read(x, c):
    rows = c["k"] or c["L"]
    here = torch.arange(rows, device=DEV)[None, :] < x["counts"][:, None]
    tables, out = _tables(), [torch.zeros_like(t) for t in x["rows"]]
    for l in range(c["layers"]):
        k, v, s = _picked(x, c, l) if c["k"] else [t[l] for t in x["cache"]]
        for j, code in enumerate((k, v)):
            val = _values(code, s[..., j, :], c["bits"], tables)
            out[j][l] = torch.where(here[..., None, None], val, torch.zeros_like(val))
    return dict(K=out[0], V=out[1])


def _attend(q, k, v, seen):
    """q [B][H_q][D], k and v [B][rows][H_kv][D] in 32 bits, seen [B][rows]: outputs and
    log-sum-exps; a query that sees nothing: 0 and -inf."""
    B, H_q, _ = q.shape
    H_kv = k.shape[2]
    q = q.float().view(B, H_kv, H_q // H_kv, D)
    s = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(D))
    s = s.masked_fill_(~seen[:, None, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = e.sum(-1, keepdim=True)
    out = torch.matmul(e, v.permute(0, 2, 1, 3).contiguous()) / torch.where(
        z == 0, torch.ones_like(z), z)
    return out.view(B, H_q, D), (m + torch.log(z)).view(B, H_q)


def _plain_attend(x, c):
    """Layer by layer; of a window, its rows alone are read."""
    tables, out, lse = _tables(), [], []
    L, W, S = c["L"], c.get("window", 0), c.get("sinks", 0)
    for l in range(c["layers"]):
        if c["kind"] == "sparse":
            k, v, s = _picked(x, c, l)
            seen = torch.arange(c["k"], device=DEV)[None, :] < x["counts"][:, None]
        elif W:
            lens = x["lens"].long()[:, None]
            j = torch.arange(min(L, W + S), device=DEV)[None, :]
            t = torch.where(j < S, j, j + torch.clamp(lens - W - S, min=0))
            seen = t < lens
            t = torch.where(seen, t, torch.zeros_like(t))
            b = torch.arange(c["B"], device=DEV)[:, None]
            k, v, s = (y[l][b, t] for y in x["cache"])
        else:
            k, v, s = (y[l] for y in x["cache"])
            seen = torch.arange(L, device=DEV)[None, :] < x["lens"][:, None]
        o, z = _attend(x["q"][l], _values(k, s[..., 0, :], c["bits"], tables),
                       _values(v, s[..., 1, :], c["bits"], tables), seen)
        out.append(o)
        lse.append(z)
    return dict(out=torch.stack(out), lse=torch.stack(lse))


# ------------------------------------------------------------------ one pass

def _own(x, c):
    """The framework's calls, with outputs and a workspace that a program keeps."""
    import paper_2512_00722_amd as spec

    kind = c["kind"]
    if "held" not in x:
        x["held"] = spec.QuantCache.of(*x["cache"])
        if "q" in x:
            dims = spec.QuantDims.make(
                B=c["B"], L_cap=c["L"], n_layers=c["layers"], H_q=c["H_q"], H_kv=c["H_kv"],
                bits=c["bits"], window=c.get("window") or c["L"], n_sink=c.get("sinks", 0),
                k_max=c.get("k", 0), n_sets=c.get("sets", 1))
            need = spec.quant_workspace_size(
                dims, spec.QUANT_DECODE if kind == "decode" else spec.QUANT_SPARSE_DECODE)
            x["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
    cache = x["held"]
    if kind == "append":
        spec.quant_append(cache, x["k_new"], x["v_new"], x["pos"], n_new=x["n_new"])
        K, V = spec.quant_read(cache, x["n_new"], idx=x["idx"], out=x["rows"])
        return dict(K=K, V=V)
    if kind == "read":
        K, V = spec.quant_read(cache, x["counts"], idx=x.get("idx"), out=x["rows"])
        return dict(K=K, V=V)
    if kind == "decode":
        out, lse = spec.quant_decode_attn(x["q"], cache, x["lens"], window=c["window"] or None,
                                          n_sink=c["sinks"], out=x["out"], lse=x["lse"],
                                          ws=x["ws"])
    else:
        out, lse = spec.quant_sparse_decode_attn(x["q"], cache, x["counts"], x["idx"],
                                                 out=x["out"], lse=x["lse"], ws=x["ws"])
    return dict(out=out, lse=lse)


def run(x):
    c = x["case"]
    if own:
        return _own(x, c)
    return dict(append=_plain_append, read=_plain_read, decode=_plain_attend,
                sparse=_plain_attend)[c["kind"]](x, c)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = dict(case)
    n, B, H_kv = c["layers"], c["B"], c["H_kv"]
    half = 0.5 if c["ragged"] else 1.0               # expected share of the longest length
    held = H_kv * 2 * (D * c["bits"] // 8 + D // GROUP)   # K and V of a token, as they are held
    wide = H_kv * 2 * D * 2                          # in bf16
    if c["kind"] == "append":
        toks = n * B * c["T"] * half
        return dict(bytes=2 * toks * (held + wide), flops=4.0 * toks * H_kv * 2 * D)
    if c["kind"] == "read":
        toks = n * B * (c["k"] or c["L"]) * half
        return dict(bytes=toks * (held + wide), flops=toks * H_kv * 2 * D)
    rows = c["k"] * half if c["kind"] == "sparse" else min(
        c["L"] * half, c["window"] + c["sinks"] if c["window"] else c["L"])
    toks = n * B * rows
    io = n * B * c["H_q"] * (D * 6 + 4)              # queries, outputs, log-sum-exps
    return dict(bytes=toks * held + io, flops=4.0 * toks * c["H_q"] * D)


# ------------------------------------------------------------------ in 64 bits

def _exact_held(x, bits):
    """What x [.., D] reads back as, from the definition: a step is the spacing of the
    elements at a magnitude, and a power of two of the group."""
    g = x.double().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    largest, low, mant = (6.0, 0, 1) if bits == 4 else (448.0, -6, 3)
    X = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / (7.0 if bits == 4 else 448.0)))
    fits = 7.0 if bits == 4 else 448.0
    X = torch.where(top <= fits * torch.exp2(X - 1), X - 1, X)   # a logarithm next to a border
    X = torch.where(top > fits * torch.exp2(X), X + 1, X).clamp(-111, 125 if bits == 4 else 119)
    y = g / torch.exp2(X)
    _, e = torch.frexp(y.abs())
    step = torch.exp2((e - 1).clamp(min=low).double() - mant)
    y = (torch.round(y / step) * step).clamp(-largest, largest) * torch.exp2(X)
    y = torch.where(torch.isfinite(top), y, torch.full_like(y, math.nan))
    return y.flatten(-2)


def _exact_values(code, scale, bits):
    """Values of held rows [.., D] from the elements' bits: sign, exponent, mantissa."""
    if bits == 4:
        e = torch.stack([code % 16, code // 16], -1).flatten(-2).double()
        sign, rest, mant, low = e >= 8, e % 8, 1, 1
    else:
        e = code.double()
        sign, rest, mant, low = e >= 128, e % 128, 3, 7
    exp = torch.floor(rest / 2 ** mant)
    frac = (rest - exp * 2 ** mant) / 2 ** mant
    mag = torch.where(exp == 0, frac * 2.0 ** (1 - low), (1 + frac) * torch.exp2(exp - low))
    power = torch.exp2(scale.double() - 127)
    return torch.where(sign, -mag, mag) * power.repeat_interleave(GROUP, -1)


def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    n, B, H_kv, bits, L = c["layers"], c["B"], c["H_kv"], c["bits"], c["L"]
    if c["kind"] == "append":
        here = torch.arange(c["T"], device=DEV)[None, :] < x["n_new"][:, None]
        res = {}
        for name, new in (("K", x["k_new"]), ("V", x["v_new"])):
            rows = torch.zeros(new.shape, dtype=torch.float32, device=DEV)
            for l in range(n):
                rows[l] = torch.where(here[..., None, None], _exact_held(new[l], bits), 0.0)
            res[name] = rows
        return res
    k, v, s = _cache(c, seed)
    if c["kind"] == "read":
        rows = c["k"] or L
        res = {m: torch.zeros((n, B, rows, H_kv, D), dtype=torch.float32, device=DEV)
               for m in "KV"}
        for l in range(n):
            for b, m in enumerate(x["counts"].tolist()):
                for h in range(H_kv):
                    t = torch.arange(m, device=DEV)
                    if c["k"]:
                        t = (x["idx"][b] if c["sets"] == 1 else x["idx"][b, h])[:m].long()
                    for j, (name, code) in enumerate((("K", k), ("V", v))):
                        res[name][l, b, :m, h] = _exact_values(code[l, b, t, h],
                                                               s[l, b, t, h, j], bits)
        return res
    q = x["q"]
    G = c["H_q"] // H_kv
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:-1], -math.inf, dtype=torch.float64, device=DEV)
    lengths = (x["lens"] if c["kind"] == "decode" else x["counts"]).tolist()
    for l in range(n):
        for b, m in enumerate(lengths):
            for h in range(H_kv):
                t = torch.arange(m, device=DEV)
                if c["kind"] == "sparse":
                    t = (x["idx"][b] if c["sets"] == 1 else x["idx"][b, h])[:m].long()
                elif c["window"]:
                    t = t[(t < c["sinks"]) | (t > m - 1 - c["window"])]
                if t.numel() == 0:
                    continue
                hs = slice(h * G, (h + 1) * G)
                kk = _exact_values(k[l, b, t, h], s[l, b, t, h, 0], bits)
                vv = _exact_values(v[l, b, t, h], s[l, b, t, h, 1], bits)
                a = q[l, b, hs].double() @ kk.t().contiguous() / math.sqrt(D)
                lse[l, b, hs] = torch.logsumexp(a, -1)
                out[l, b, hs] = torch.softmax(a, -1) @ vv
    return dict(out=out, lse=lse)
