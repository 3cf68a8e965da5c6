"""Strided tensors through the binding's native marshalling: what it must leave to
the wrapper's checks, which raise before anything is launched."""
import pytest
import torch

import paper_2512_00722_amd as spec
from tests import strided_calls
from tests.gpu_helpers import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return need_gpu()


@pytest.mark.parametrize("name", strided_calls.NAMES)
def test_expanded_tensors_are_refused(dev, name):
    announce(f"expanded tensors, {name}")
    a = strided_calls.tensors(dev)
    strided, plain = strided_calls.calls(a)[name]
    for pair in (("K", "V"), ("K_prefix", "V_prefix"), ("K_r",), ("ckv",)):
        for dim in range(2 if pair[0] in ("K", "ckv") else 1):
            if pair[0] not in strided:
                continue
            b = dict(a)
            for t in pair:
                b[t] = strided_calls.expanded(a[t], dim)
            with pytest.raises(ValueError, match="expanded"):
                strided_calls.calls(b)[name][1]()
    plain()    # the tensors themselves are fine
    torch.cuda.synchronize()


def test_strides_of_single_entries_mean_nothing(dev):
    """One layer and one sequence whose strides are arbitrary, with every buffer handed
    over and without: the results of the packed tensors."""
    announce("strides of single entries")
    g = torch.Generator(device=dev).manual_seed(3)

    def rn(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    K, V, Kp, Vp = rn(1, 1, 90, 2, 128), rn(1, 1, 90, 2, 128), rn(1, 70, 2, 128), rn(1, 70, 2, 128)
    q, qc = rn(1, 1, 8, 128), rn(1, 1, 6, 8, 128)
    lens = torch.tensor([83], dtype=torch.int32, device=dev)
    idx = torch.arange(0, 64, 2, dtype=torch.int32, device=dev)[None]
    n = torch.tensor([32], dtype=torch.int32, device=dev)
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device=dev)

    def outputs(t, kind=torch.float32):
        return dict(out=torch.zeros(t.shape, dtype=kind, device=dev),
                    lse=torch.zeros(t.shape[:-1], device=dev), ws=ws)

    def run(K, V, Kp, Vp, buffers):
        o = (lambda t, *k: outputs(t, *k)) if buffers else (lambda t, *k: {})
        w = torch.zeros((1, 1, 1, 90), device=dev)
        return [*spec.window_decode_attn(q, K, V, lens, 30, **o(q)),
                *spec.window_attn(qc, K, V, lens, 30, **o(qc, torch.bfloat16)),
                *spec.prefix_decode_attn(q, Kp, Vp, K, V, lens, **o(q)),
                *spec.accum_decode_attn(q, K, V, lens, w, **o(q)), w,
                *spec.sparse_decode_attn(q, K, V, n, idx=idx, **o(q))]

    want = run(K, V, Kp, Vp, True)
    kv = [strided_calls.loose(strided_calls.loose(t, 0), 1) for t in (K, V)]
    pre = [strided_calls.loose(t, 0) for t in (Kp, Vp)]
    for buffers in (True, False):
        for a, b in zip(run(*kv, *pre, buffers), want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", [n for n in strided_calls.NAMES if n != "gather"])
def test_workspaces_are_whole_device_memory(dev, name):
    announce(f"workspace views, {name}")
    a = strided_calls.tensors(dev)
    for ws in (a["ws"][:1].expand(1 << 24), a["ws"][::2], torch.zeros(1 << 24, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="ws must be"):
            strided_calls.calls(dict(a, ws=ws))[name][1]()
