"""The outputs that spec.quant_read takes: two tensors, nothing else (nothing is launched)."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2512_00722_amd as spec

N, B, L, H, D, K = 2, 3, 40, 2, 128, 16


@pytest.mark.parametrize("with_idx", (False, True))
@pytest.mark.parametrize("make", [
    lambda k, v: (k, v, v), lambda k, v: (k,), lambda k, v: (), lambda k, v: (k, None),
    lambda k, v: (None, v), lambda k, v: (None, None), lambda k, v: [k, v, None]],
    ids=["three", "one", "none", "no V", "no K", "neither", "three in a list"])
def test_outputs_are_two_tensors(make, with_idx):
    with FakeTensorMode():
        def rows():
            return torch.zeros((N, B, K, H, D), dtype=torch.bfloat16, device="cuda")

        cache = spec.QuantCache(N, B, L, H, device="cuda")
        counts = torch.zeros(B, dtype=torch.int32, device="cuda")
        idx = torch.zeros((B, K), dtype=torch.int32, device="cuda") if with_idx else None
        with pytest.raises(ValueError, match="out must be"):
            spec.quant_read(cache, counts, idx=idx, out=make(rows(), rows()))
