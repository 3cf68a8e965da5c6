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
