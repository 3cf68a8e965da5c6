"""Caches held in 4 or 8 bits on a host without a GPU: the oracle against the definition,
and what the C ABI and the binding refuse (nothing is launched)."""
import ctypes
import math

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2512_00722_amd as spec
from oracle import quant_oracle as qo

FAKE = 0x7000_0000_0000       # 16-byte aligned, never dereferenced
APPEND, READ, DECODE, SPARSE = range(4)


# ------------------------------------------------------------------ the oracle

def test_the_elements():
    assert qo.elements(4).tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4,
                                       -6]
    e = qo.elements(8)
    want = torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(e, want)
    assert np.nanmax(e) == 448 and e[1] == 2.0 ** -9


@pytest.mark.parametrize("bits,fits,largest", [(4, 7.0, 6.0), (8, 448.0, 448.0)])
def test_the_scales(bits, fits, largest):
    """The least power of two that the group fits; what does not round within the elements
    saturates; groups of zeros and NaNs; the clamped ends."""
    x = np.zeros((9, 32))
    x[0, 3] = -fits                       # fits 2^0
    x[1, 3] = fits * (1 + 2.0 ** -7)      # does not
    x[2, 3] = fits * 2.0 ** -20
    x[4, 3] = math.nan
    x[5, 3] = -math.inf
    x[6, 3] = 2.0 ** -133                 # the least bf16
    x[7, 3] = (2 - 2.0 ** -7) * 2.0 ** 127   # the largest
    x[8, 3] = fits * 2.0 ** -111
    codes, scales = qo.quantise(x, bits)
    most = {4: 125, 8: 119}[bits]
    assert (scales[:, 0].astype(int) - 127).tolist() == [0, 1, -20, -111, 128, 128, -111, most,
                                                         -111]
    v = qo.values(codes, scales, bits)
    assert v[0, 3] == -largest and np.isnan(v[4:6]).all()
    assert v[6, 3] == 0 and v[3, 3] == 0
    assert v[7, 3] == largest * 2.0 ** most      # saturated


@pytest.mark.parametrize("bits", [4, 8])
def test_no_element_is_off_by_more_than_half_a_step(bits):
    g = np.random.default_rng(1)
    x = g.standard_normal((4000, 128)) * np.exp2(g.integers(-20, 20, (4000, 1)))
    x = torch.tensor(x).to(torch.bfloat16).double().numpy()
    codes, scales = qo.quantise(x, bits)
    v = qo.values(codes, scales, bits)
    grid = np.sort(qo.elements(bits)[np.isfinite(qo.elements(bits))])
    y = x / np.repeat(np.exp2(scales.astype(float) - 127), 32, -1)
    near = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
    best = np.minimum(np.abs(y - grid[near]), np.abs(y - grid[near - 1]))
    got = np.abs(v / np.repeat(np.exp2(scales.astype(float) - 127), 32, -1) - y)
    np.testing.assert_array_equal(got, best)
    top = grid[-1] - grid[-2]
    assert (got <= np.where(np.abs(y) > grid[-2], top / 2, top / 2)).all()
    assert (v == torch.tensor(v).to(torch.bfloat16).double().numpy()).all()
    # a step of scale more coarse would hold the group too, one less would not
    amax = np.abs(x).reshape(-1, 32).max(-1)
    X = scales.reshape(-1).astype(float) - 127
    fits = qo.FORMATS[bits][2]
    assert (amax <= fits * np.exp2(X)).all() and (amax > fits * np.exp2(X - 1)).all()


def test_ties_go_to_the_even_element():
    x = np.zeros((1, 32))
    x[0, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    codes, scales = qo.quantise(x, 4)
    assert scales[0, 0] == 127
    assert qo.values(codes, scales, 4)[0, :8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4]
    assert qo.unpack(qo.pack(codes, 4), 4).tolist() == codes.tolist()


# ------------------------------------------------------------------ the C ABI

@pytest.fixture(scope="module")
def lib():
    return spec.load_library()


def dims(**kw):
    base = dict(B=2, L_cap=4096, n_layers=2, H_q=32, H_kv=8, d=128, bits=4, T=5, window=4096,
                n_sink=0, k_max=512, n_sets=1)
    base.update(kw)
    return spec.QuantDims.make(**base)


def size(lib, d, op):
    n = ctypes.c_size_t(0)
    return lib.spec_quant_workspace_size(ctypes.byref(d), op, ctypes.byref(n)), n.value


def call(lib, op, d, cache=(FAKE, FAKE, FAKE), ptrs=None, ws=FAKE, nws=1 << 40):
    """The entry point `op` with fake pointers (never dereferenced: the checks come first)."""
    c = spec.QuantBuffers(*cache)
    P = [ctypes.c_void_p(p) for p in (ptrs or (FAKE,) * 4)]
    if op == APPEND:
        return lib.spec_quant_append(ctypes.byref(d), ctypes.byref(c), *P[:4], None)
    if op == READ:
        return lib.spec_quant_read(ctypes.byref(d), ctypes.byref(c), *P[:4], None)
    if op == DECODE:
        return lib.spec_quant_decode_attn(ctypes.byref(d), P[0], ctypes.byref(c), P[1], P[2], P[3],
                                          ctypes.c_void_p(ws), nws, None)
    P += [ctypes.c_void_p(FAKE)]
    return lib.spec_quant_sparse_decode_attn(ctypes.byref(d), P[0], ctypes.byref(c), P[1], P[2],
                                             P[3], P[4], ctypes.c_void_p(ws), nws, None)


@pytest.mark.parametrize("field,value,status,ops", [
    ("B", 0, 1, range(4)), ("L_cap", -1, 1, range(4)), ("n_layers", 0, 1, range(4)),
    ("H_kv", 0, 1, range(4)), ("d", 0, 1, range(4)), ("d", 64, 2, range(4)),
    ("bits", 5, 2, range(4)), ("bits", 0, 2, range(4)), ("reserved", 1, 1, range(4)),
    ("scale", -1.0, 1, range(4)), ("scale", math.nan, 1, range(4)),
    ("H_q", 30, 1, (DECODE, SPARSE)), ("H_q", 0, 1, (DECODE, SPARSE)),
    ("H_q", 8 * 129, 2, (DECODE, SPARSE)),
    ("T", 0, 1, (APPEND,)), ("window", 0, 1, (DECODE,)), ("n_sink", -1, 1, (DECODE,)),
    ("k_max", 0, 1, (READ, SPARSE)), ("k_max", 4097, 1, (READ, SPARSE)),
    ("n_sets", 2, 2, (READ, SPARSE)), ("n_sets", 0, 2, (READ, SPARSE)),
    ("kv_stride_b", 4096 * 8 * 64 - 16, 1, range(4)), ("kv_stride_b", 4096 * 8 * 64 + 8, 1, range(4)),
    ("kv_stride_layer", -16, 1, range(4)), ("kv_stride_layer", 16, 1, range(4)),
    ("scale_stride_b", 4096 * 64 - 8, 1, range(4)), ("scale_stride_b", 4096 * 64 + 4, 1, range(4)),
    ("scale_stride_layer", 8, 1, range(4)),
    ("B", 65536, 2, range(4)), ("n_layers", 65536, 2, range(4)), ("H_kv", 65536, 2, (APPEND,)),
    ("L_cap", (1 << 30) + 1, 2, (APPEND, DECODE)), ("T", (1 << 30) + 1, 2, (APPEND,)),
])
def test_dims_are_checked(lib, field, value, status, ops):
    d = dims()
    setattr(d, field, value)
    for op in ops:
        assert size(lib, d, op)[0] == status, (field, op)
        assert call(lib, op, d) == status, (field, op)
    assert lib.spec_last_hip_error() == 0


def test_the_documented_limits(lib):
    """At them and beyond (the sizing validates as the calls do)."""
    big = dict(n_layers=64, B=32768, H_kv=1, H_q=1, L_cap=64, k_max=64, window=64)
    for op in range(4):
        assert size(lib, dims(**big), op)[0] == 0
        assert size(lib, dims(**{**big, "n_layers": 65}), op)[0] == 2
    for op in (DECODE, SPARSE):
        for at, beyond in ((dict(big, H_q=32), dict(H_q=33)),                    # 2^26 rows
                           (dict(big, n_layers=4, B=30840, H_q=34, H_kv=2), dict(B=30841))):
            assert size(lib, dims(**at), op)[0] == 0
            assert size(lib, dims(**{**at, **beyond}), op)[0] == 2
    one = dict(n_layers=1, B=1, H_kv=1, L_cap=1 << 28)
    n = (1 << 28) - 16
    assert size(lib, dims(**one, k_max=n), READ)[0] == 0
    assert size(lib, dims(**one, k_max=n + 1), READ)[0] == 2
    assert size(lib, dims(**one, T=n), APPEND)[0] == 0
    assert size(lib, dims(**one, T=n + 1), APPEND)[0] == 2
    assert size(lib, dims(n_layers=1, B=1, H_kv=1, H_q=1, L_cap=1 << 30, window=1 << 30),
                DECODE)[0] == 0


@pytest.mark.parametrize("op", range(4))
def test_pointers_are_checked(lib, op):
    d = dims()
    need = size(lib, d, op)[1]
    for i in range(3):
        for bad in (0, FAKE + (4 if i == 2 else 8)):
            c = [FAKE] * 3
            c[i] = bad
            assert call(lib, op, d, cache=c, nws=max(need, 16)) == 1
    optional = {APPEND: (3,), READ: (0,), DECODE: (3,), SPARSE: ()}[op]
    for i in range(4):
        if i not in optional:
            p = [FAKE] * 4
            p[i] = 0
            assert call(lib, op, d, ptrs=p, nws=max(need, 16)) == 1
        p = [FAKE] * 4
        p[i] = FAKE + 2
        assert call(lib, op, d, ptrs=p, nws=max(need, 16)) == 1
    assert lib.spec_quant_append(ctypes.byref(d), None, *[ctypes.c_void_p(FAKE)] * 4, None) == 1
    if need:
        assert call(lib, op, d, nws=need - 1) == 3
        assert call(lib, op, d, ws=0, nws=need) == 3
        assert call(lib, op, d, ws=FAKE + 8, nws=need) == 1
    assert lib.spec_last_hip_error() == 0


def test_workspace_sizes(lib):
    for op in (APPEND, READ):
        assert size(lib, dims(), op) == (0, 0)
    assert size(lib, dims(), 4)[0] == 1 and size(lib, dims(), -1)[0] == 1
    assert lib.spec_quant_workspace_size(ctypes.byref(dims()), DECODE, None) == 1
    st, n = size(lib, dims(B=1, n_layers=1), DECODE)
    assert st == 0 and n >= 2 * 32 * 130 * 4 and n % 256 == 0     # in parts
    assert size(lib, dims(B=64, n_layers=32, window=512), DECODE) == (0, 0)   # enough without
    assert size(lib, dims(B=64, n_layers=32), SPARSE) == (0, 0)
    # one device's plan for every device: the same size however often it is asked
    assert size(lib, dims(B=1, n_layers=1), DECODE)[1] == n


def test_plans_of_all_sizes(lib):
    """Sizing takes any shape within the limits (a plan exists), and a split is never of more
    parts than there are chunks of 32 tokens: at most rows x ceil(tokens / 32) partial results
    of 130 floats, in two regions of whole 256 bytes, and 512 for where up to 64 sequences'
    parts begin."""
    rng = np.random.default_rng(5)
    for _ in range(3000):
        H_kv = int(rng.integers(1, 17))
        G = int(rng.integers(1, 129))
        n, B = (int(2 ** rng.uniform(0, 6)) for _ in range(2))
        cap = int(2 ** rng.uniform(0, 20))
        k = int(rng.integers(1, cap + 1))
        w, sink = int(2 ** rng.uniform(0, 21)), int(rng.integers(0, 64))
        d = dims(B=B, n_layers=n, L_cap=cap, H_kv=H_kv, H_q=G * H_kv, k_max=k, window=w,
                 n_sink=sink, bits=int(rng.choice([4, 8])), n_sets=int(rng.choice([1, H_kv])))
        for op, tokens in ((DECODE, min(cap, w + sink)), (SPARSE, k)):
            st, need = size(lib, d, op)
            assert st == 0
            assert need <= n * B * H_kv * G * -(-tokens // 32) * 130 * 4 + 1024


# ------------------------------------------------------------------ the binding

N, B, L, H, D, T, K = 2, 3, 40, 2, 128, 5, 16


def tensors(bits=4, device="cuda"):
    def u8(*s):
        return torch.zeros(s, dtype=torch.uint8, device=device)

    def bf(*s):
        return torch.zeros(s, dtype=torch.bfloat16, device=device)

    def i32(*s):
        return torch.zeros(s, dtype=torch.int32, device=device)

    w = 16 * bits
    return dict(k=u8(N, B, L, H, w), v=u8(N, B, L, H, w), s=u8(N, B, L, H, 2, 4),
                k_new=bf(N, B, T, H, D), v_new=bf(N, B, T, H, D), pos=i32(B), n_new=i32(B),
                counts=i32(B), idx=i32(B, K), q=bf(N, B, 4 * H, D),
                out=torch.zeros((N, B, 4 * H, D), device=device),
                lse=torch.zeros((N, B, 4 * H), device=device),
                rows=(bf(N, B, K, H, D), bf(N, B, K, H, D)), ws=u8(1 << 22))


def calls(a):
    c = spec.QuantCache.of(a["k"], a["v"], a["s"])
    o = dict(out=a["out"], lse=a["lse"], ws=a["ws"])
    return dict(
        append=lambda: spec.quant_append(c, a["k_new"], a["v_new"], a["pos"], n_new=a["n_new"]),
        read=lambda: spec.quant_read(c, a["counts"], idx=a["idx"], out=a["rows"]),
        decode=lambda: spec.quant_decode_attn(a["q"], c, a["counts"], **o),
        sparse=lambda: spec.quant_sparse_decode_attn(a["q"], c, a["counts"], a["idx"], **o))


def test_caches():
    for bits in (4, 8):
        c = spec.QuantCache(N, B, L, H, bits=bits, device="cpu")
        assert c.bits == bits and c.k.shape == (N, B, L, H, 16 * bits) and c.device.type == "cpu"
        assert c.scales.shape == (N, B, L, H, 2, 4) and not c.k.any() and not c.scales.any()
        part = c.layers(1, 2)
        assert part.k.data_ptr() == c.k[1].data_ptr() and part.k.shape[0] == 1
        with pytest.raises(AttributeError):
            c.k = c.v
        with pytest.raises(ValueError, match="device"):
            spec.quant_read(c, torch.zeros(B, dtype=torch.int32))
    for kw in (dict(bits=5), dict(d=64)):
        with pytest.raises(ValueError):
            spec.QuantCache(N, B, L, H, device="cpu", **kw)


@pytest.mark.parametrize("name,make,error,match", [
    ("k", lambda a: a["k"].to(torch.int8), TypeError, "uint8"),
    ("v", lambda a: a["v"][..., :32], ValueError, "same shape"),
    ("k", lambda a: a["k"][0], ValueError, "5 dims"),
    ("s", lambda a: a["s"][:, :, :-1], ValueError, "scales"),
    ("s", lambda a: a["s"][..., :2], ValueError, "scales"),
    ("s", lambda a: a["s"][:, :, :, :, :, :1].expand(-1, -1, -1, -1, -1, 4), ValueError,
     "contiguous"),
    ("k", lambda a: "k", TypeError, "tensor"),
    ("s", lambda a: a["s"].cpu(), ValueError, "must be on"),
])
def test_caches_that_are_refused(name, make, error, match):
    with FakeTensorMode():
        a = tensors()
        a[name] = make(a)
        with pytest.raises(error, match=match):
            calls(a)


def test_strided_caches():
    with FakeTensorMode():
        a = tensors()
        for dim in (0, 1):
            shape = list(a["k"].shape)
            b = dict(a)
            for t in ("k", "v"):
                b[t] = a[t].narrow(dim, 0, 1).expand(shape)
            with pytest.raises(ValueError, match="expanded"):
                calls(b)
            b = dict(a, s=a["s"].narrow(dim, 0, 1).expand(a["s"].shape))
            with pytest.raises(ValueError, match="expanded"):
                calls(b)
        b = dict(a)
        for t in ("k", "v"):
            b[t] = a[t].transpose(2, 3).contiguous().transpose(2, 3)
        with pytest.raises(ValueError, match="contiguous"):
            calls(b)


@pytest.mark.parametrize("call_name,name,make,error,match", [
    ("append", "k_new", lambda t: t.float(), TypeError, "bfloat16"),
    ("append", "v_new", lambda t: t[:, :, :-1], ValueError, "v_new"),
    ("append", "k_new", lambda t: t.transpose(0, 1), ValueError, "k_new"),
    ("append", "k_new", lambda t: t[0], (TypeError, ValueError), "k_new"),
    ("append", "pos", lambda t: t.long(), TypeError, "int32"),
    ("append", "pos", lambda t: t[:-1], ValueError, "pos"),
    ("append", "n_new", lambda t: t.cpu(), ValueError, "n_new"),
    ("read", "counts", lambda t: t[:-1], ValueError, "counts"),
    ("read", "idx", lambda t: t.long(), TypeError, "int32"),
    ("read", "idx", lambda t: t[:-1], ValueError, "idx"),
    ("read", "idx", lambda t: t[:, ::2], ValueError, "idx"),
    ("read", "idx", lambda t: t[:, None].expand(B, H + 1, K), ValueError, "H_kv"),
    ("read", "rows", lambda t: (t[0], t[1].float()), TypeError, "bfloat16"),
    ("read", "rows", lambda t: (t[0][:, :, :-1], t[1]), ValueError, "K must be"),
    ("decode", "q", lambda t: t.float(), TypeError, "bfloat16"),
    ("decode", "q", lambda t: t[:1], ValueError, "q must be"),
    ("decode", "q", lambda t: t.transpose(0, 1), ValueError, "q must be"),
    ("decode", "counts", lambda t: t.float(), TypeError, "int32"),
    ("decode", "out", lambda t: t.half(), TypeError, "float32"),
    ("decode", "out", lambda t: t[:, :, :-1], ValueError, "out"),
    ("decode", "lse", lambda t: t[..., None], ValueError, "lse"),
    ("decode", "ws", lambda t: t[::2], ValueError, "ws must be"),
    ("decode", "ws", lambda t: t[:1].expand(1 << 24), ValueError, "ws must be"),
    ("sparse", "q", lambda t: t.float(), TypeError, "bfloat16"),
    ("sparse", "idx", lambda t: t[0], ValueError, "idx"),
    ("sparse", "idx", lambda t: t.cpu(), ValueError, "device"),
    ("sparse", "counts", lambda t: t[:-1], ValueError, "counts"),
    ("sparse", "ws", lambda t: t.cpu(), ValueError, "ws must be"),
])
def test_arguments_that_are_refused(call_name, name, make, error, match):
    with FakeTensorMode():
        a = tensors()
        a[name] = make(a[name])
        with pytest.raises(error, match=match):
            calls(a)[call_name]()


def test_a_cache_is_a_quant_cache():
    with FakeTensorMode():
        a = tensors()
        for f in (lambda: spec.quant_append((a["k"], a["v"], a["s"]), a["k_new"], a["v_new"],
                                            a["pos"]),
                  lambda: spec.quant_read(a["k"], a["counts"]),
                  lambda: spec.quant_decode_attn(a["q"], a["k"], a["counts"]),
                  lambda: spec.quant_sparse_decode_attn(a["q"], a["k"], a["counts"], a["idx"])):
            with pytest.raises(TypeError, match="QuantCache"):
                f()
