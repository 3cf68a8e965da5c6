"""The entry points over caches that are read in full, where arguments share memory."""
import pytest
import torch

import paper_2512_00722_amd as spec
from tests.gpu_helpers import announce
from tests.test_dense_gpu import D, bounded, dev, evict_reference, i32, normal, same_bits

pytestmark = pytest.mark.gpu
assert dev  # the fixture


# ------------------------------------------------------------------ eviction

@pytest.mark.parametrize("T,cap", [(30, 100), (40, 100), (30, 40000)])
@pytest.mark.parametrize("alias", ["n_new", "keep"])
def test_evict_arguments_in_the_counts(dev, T, cap, alias):
    """The new rows, or the budgets, read from the tensor of the counts, which the call
    rewrites."""
    announce(f"evict {alias} in the counts, {T} {cap}")
    n, B, H_kv = 2, 3, 2
    counts = [20, cap, 25] if alias == "n_new" else [20, 60, 0]
    rows = [min(c, T) for c in counts] if alias == "n_new" else [T, 7, 2]
    keep = [35, 60, 40] if alias == "n_new" else counts
    x = bounded(n, B, H_kv, H_kv, cap, 301, dev)
    x[3][:, 0] = torch.randperm(cap, generator=torch.Generator().manual_seed(302)).int().to(dev)
    x[3][:, 0, :, :20] = torch.arange(180, 200, dtype=torch.int32).flip(0).to(dev)
    pos = [200, 3 * cap, 50]
    k_new, v_new = (normal((n, B, T, H_kv, D), 303 + i, dev) for i in range(2))
    *want, after = evict_reference(x, H_kv, counts, keep, pos, rows, k_new, v_new, 25, 2)
    c = i32(counts, dev)
    spec.evict(*x, c, c if alias == "keep" else i32(keep, dev), i32(pos, dev), k_new=k_new,
               v_new=v_new, n_new=c if alias == "n_new" else i32(rows, dev), n_recent=25, n_sink=2)
    torch.cuda.synchronize()
    assert c.tolist() == after
    for got, ref, nm in zip(x, want, ("K", "V", "weights", "tokens")):
        assert same_bits(got, ref), nm
