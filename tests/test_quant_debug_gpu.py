"""SPEC_DEBUG over caches in 4 and 8 bits: a sequence without new rows has none outside the
caches, wherever its position stands."""
import pytest
import torch

import paper_2512_00722_amd as spec
from tests.gpu_helpers import announce, need_gpu
from tests.quant_helpers import D, held, i32, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", (4, 8))
@pytest.mark.parametrize("pos", (-1, -7, 33, 1 << 30, -(1 << 31)))
def test_idle_sequences(bits, pos, monkeypatch):
    dev = need_gpu()
    announce(f"idle sequence at {pos} {bits}")
    n, B, cap, H_kv, T = 2, 3, 32, 2, 4
    k_new, v_new = (normal((n, B, T, H_kv, D), 801 + i, dev) for i in range(2))
    plain, debug = (held((n, B, cap, H_kv), 803, bits, dev) for _ in range(2))
    args = k_new, v_new, i32([3, pos, 28], dev)
    spec.quant_append(plain, *args, n_new=i32([2, 0, 4], dev))
    monkeypatch.setenv("SPEC_DEBUG", "1")
    spec.quant_append(debug, *args, n_new=i32([2, 0, 4], dev))
    for a, b in zip((plain.k, plain.v, plain.scales), (debug.k, debug.v, debug.scales)):
        assert torch.equal(a, b)
    for n_new in ([2, 1, 4], [2, 0, 5]):
        with pytest.raises(spec.SpecError):
            spec.quant_append(debug, *args, n_new=i32(n_new, dev))
    with pytest.raises(spec.SpecError):
        spec.quant_append(debug, *args)
