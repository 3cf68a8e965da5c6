"""Strided tensors that a call must refuse, on a host without a GPU (tensors without
memory: nothing is launched)."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2512_00722_amd as spec
from tests import strided_calls


@pytest.mark.parametrize("name", strided_calls.NAMES)
def test_expanded_tensors_are_refused(name):
    """A stride of 0 means 'densely packed' to the library, which would go past the
    tensor's memory."""
    with FakeTensorMode():
        a = strided_calls.tensors("cuda")
        strided = strided_calls.calls(a)[name][0]
        pairs = [p for p in (("K", "V"), ("K_prefix", "V_prefix"), ("K_r",), ("ckv",))
                 if p[0] in strided]
        seen = 0
        for pair in pairs:
            outer = 2 if pair[0] in ("K", "ckv") else 1
            for dim in range(outer):
                b = dict(a)
                for t in pair:
                    b[t] = strided_calls.expanded(a[t], dim)
                    assert b[t].stride(dim) == 0
                with pytest.raises(ValueError, match="expanded"):
                    strided_calls.calls(b)[name][1]()
                seen += 1
        assert seen


def test_expanded_host_caches_are_refused(monkeypatch):
    K = torch.zeros((1, 2, 40, 2, 128), dtype=torch.bfloat16)
    monkeypatch.setattr(torch.Tensor, "is_pinned", lambda t: True)
    spec._host_kv(K, K)
    E = strided_calls.expanded(K, 1)
    with pytest.raises(ValueError, match="expanded"):
        spec._host_kv(E, E)


def test_strides_of_single_entries_mean_nothing():
    """One layer, or one sequence: whatever torch leaves as its stride (here 8, as a
    transposed view of other sizes may have) is not passed on."""
    for shape, dim in (((1, 3, 40, 2, 128), 0), ((2, 1, 40, 2, 128), 1), ((1, 1, 40, 2, 128), 1)):
        K = strided_calls.loose(torch.zeros(shape, dtype=torch.bfloat16), dim)
        q = torch.zeros((*shape[:2], 8, 128), dtype=torch.bfloat16)
        for op in range(5):
            spec.dense_workspace_size(
                spec._dense_dims(K, H_q=8, window=8, P_cap=40, n_sets=2), op)
        spec.workspace_size(spec._dims_llm(q, K, 16, 0.0), spec.OP_ATTN)
    K_r = strided_calls.loose(torch.zeros((1, 40, 8, 64), dtype=torch.bfloat16), 0)
    spec.workspace_size(spec._dims_retrieval(K_r, 40, 16, 0.0), spec.OP_SCORE)


@pytest.mark.parametrize("name", [n for n in strided_calls.NAMES if n != "gather"])
def test_workspaces_are_whole_device_memory(name):
    """A strided or expanded view holds fewer bytes than it counts, and a host tensor
    none that a kernel may touch."""
    with FakeTensorMode():
        a = strided_calls.tensors("cuda")
        for ws in (a["ws"][:1].expand(1 << 24), a["ws"][::2],
                   torch.zeros(1 << 24, dtype=torch.uint8)):
            b = dict(a, ws=ws)
            with pytest.raises(ValueError, match="ws must be"):
                strided_calls.calls(b)[name][1]()
