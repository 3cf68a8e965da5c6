"""Every entry point of the binding that takes strided tensors, as calls on small
tensors with one of them replaced."""
import torch

import paper_2512_00722_amd as spec

N, B, L, H, D, H_R, D_R, T, K_MAX = 2, 3, 40, 2, 128, 8, 64, 5, 16
D_C, D_ROPE, D_NOPE, D_V, M_HEADS = 512, 64, 128, 128, 64


def tensors(device):
    """Arguments of every call, outputs and workspace among them."""
    def bf(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device=device)

    def i32(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=device)

    def f32(*shape):
        return torch.zeros(shape, device=device)

    a = dict(K=bf(N, B, L, H, D), K_prefix=bf(N, L, H, D), K_r=bf(B, L, H_R, D_R),
             ckv=bf(N, B, L, D_C + D_ROPE), q=bf(N, B, 4 * H, D), qc=bf(N, B, T, 4 * H, D),
             q_r=bf(B, H_R, D_R), lens=i32(B), idx=i32(B, K_MAX), weights=f32(N, B, H, L),
             tokens=i32(N, B, H, L), k_new=bf(N, B, T, H, D), out=f32(N, B, 4 * H, D),
             lse=f32(N, B, 4 * H), outc=bf(N, B, T, 4 * H, D), lsec=f32(N, B, T, 4 * H),
             scores=f32(B, L), ids=i32(B), emb=bf(10, 512), w=bf(H_R * D_R, 512),
             mq=bf(N, B, M_HEADS, D_NOPE + D_ROPE), w_uk=bf(N, M_HEADS, D_NOPE, D_C),
             w_uv=bf(N, M_HEADS, D_V, D_C), mout=f32(N, B, M_HEADS, D_V), mlse=f32(N, B, M_HEADS),
             ws=torch.zeros(1 << 24, dtype=torch.uint8, device=device))
    a["V"], a["V_prefix"] = torch.zeros_like(a["K"]), torch.zeros_like(a["K_prefix"])
    a["step"] = dict(idx=a["idx"], counts=i32(B), out=a["out"], lse=None, scores=None)
    return a


def calls(a):
    """name -> (the strided tensors it takes, the call with every buffer handed over)."""
    o = dict(out=a["out"], lse=a["lse"], ws=a["ws"])
    kv = ("K", "V")
    return {
        "window_decode_attn": (kv, lambda: spec.window_decode_attn(
            a["q"], a["K"], a["V"], a["lens"], 8, **o)),
        "window_attn": (kv, lambda: spec.window_attn(
            a["qc"], a["K"], a["V"], a["lens"], 8, out=a["outc"], lse=a["lsec"], ws=a["ws"])),
        "prefix_decode_attn": (kv + ("K_prefix", "V_prefix"), lambda: spec.prefix_decode_attn(
            a["q"], a["K_prefix"], a["V_prefix"], a["K"], a["V"], a["lens"], **o)),
        "accum_decode_attn": (kv, lambda: spec.accum_decode_attn(
            a["q"], a["K"], a["V"], a["lens"], a["weights"], **o)),
        "evict": (kv, lambda: spec.evict(
            a["K"], a["V"], a["weights"], a["tokens"], a["lens"], a["lens"], a["lens"],
            a["k_new"], a["k_new"], ws=a["ws"])),
        "sparse_decode_attn": (kv, lambda: spec.sparse_decode_attn(
            a["q"], a["K"], a["V"], a["lens"], idx=a["idx"], **o)),
        "gather": (kv, lambda: spec.gather(a["K"], a["V"], a["idx"], a["lens"])),
        "delta_gather": (kv, lambda: spec.delta_gather(
            a["idx"], a["lens"], a["K"], a["V"],
            spec.ElasticState(N, B, K_MAX, H, D, a["K"].device), ws=a["ws"])),
        "score": (("K_r",), lambda: spec.score(a["q_r"], a["K_r"], a["lens"], out=a["scores"],
                                               ws=a["ws"])),
        "step": (kv + ("K_r",), lambda: spec.step(
            a["q_r"], a["K_r"], a["lens"], a["lens"], a["q"], a["K"], a["V"], K_MAX,
            outputs=a["step"], ws=a["ws"])),
        "retrieval_qk": (("K_r",), lambda: spec.retrieval_qk(
            a["ids"], a["ids"], a["emb"], a["w"], a["w"], a["K_r"], q_r=a["q_r"], ws=a["ws"])),
        "mla_sparse_decode_attn": (("ckv",), lambda: spec.mla_sparse_decode_attn(
            a["mq"], a["ckv"], a["w_uk"], a["w_uv"], a["idx"], a["lens"], out=a["mout"],
            lse=a["mlse"], ws=a["ws"])),
    }


NAMES = ["window_decode_attn", "window_attn", "prefix_decode_attn", "accum_decode_attn", "evict",
         "sparse_decode_attn", "gather", "delta_gather", "score", "step", "retrieval_qk",
         "mla_sparse_decode_attn"]


def expanded(t, dim):
    """A view of t's shape whose `dim` repeats its first entry."""
    return t.narrow(dim, 0, 1).expand(t.shape)


def loose(t, dim):
    """t, which has one entry in `dim`, with another stride there."""
    strides = list(t.stride())
    strides[dim] = 8
    return t.as_strided(t.shape, strides)
