"""The sizes that the entry points over caches read in full take, and those beyond a
launch, on a host without a GPU."""
import ctypes

import pytest

import paper_2512_00722_amd as spec

WINDOW_DECODE, WINDOW, PREFIX, ACCUM, EVICT = range(5)


def status(op, **kw):
    base = dict(B=1, L_cap=64, n_layers=1, H_q=8, H_kv=8, T=1, window=64, P_cap=64, n_sets=1)
    base.update(kw)
    n = ctypes.c_size_t(0)
    d = spec.DenseDims.make(**base)
    return spec.load_library().spec_dense_workspace_size(ctypes.byref(d), op, ctypes.byref(n))


def test_accumulated_weights_of_all_that_fits_a_card():
    """32 layers x 32 sequences x 65536 tokens, a weight sum per KV head (256 GiB of K and V),
    whatever number of query heads share one; and the same with one sum."""
    for G in (1, 2, 4, 7, 16, 32):
        big = dict(n_layers=32, B=32, L_cap=65536, H_kv=8, H_q=8 * G)
        for n_sets in (1, 8):
            assert status(ACCUM, n_sets=n_sets, **big) == 0
    assert status(ACCUM, n_layers=32, B=32, L_cap=65537, H_kv=8, H_q=32, n_sets=8) == 2
    assert status(ACCUM, B=1, n_layers=1, H_q=1, H_kv=1, L_cap=1 << 29) == 0


@pytest.mark.parametrize("op,at,beyond", [
    (WINDOW_DECODE, dict(n_layers=64, B=32768, H_q=1, H_kv=1), dict(n_layers=65)),
    (EVICT, dict(n_layers=64, B=32768, H_q=1, H_kv=1), dict(B=32769)),
    (WINDOW, dict(n_layers=32, B=8, H_q=32, H_kv=8, T=8192), dict(T=8193)),
    (PREFIX, dict(n_layers=64, B=32768, H_q=32, H_kv=1), dict(H_q=33)),       # 2^26 rows
    (WINDOW_DECODE, dict(n_layers=4, B=30840, H_q=34, H_kv=2), dict(B=30841)),  # 17: a group each
    (WINDOW_DECODE, dict(L_cap=2 ** 31 - 4098), dict(L_cap=2 ** 31 - 4097)),
    (PREFIX, dict(P_cap=2 ** 31 - 4097), dict(P_cap=2 ** 31 - 4096)),
    (WINDOW_DECODE, dict(B=65535), dict(B=65536)),
    (WINDOW_DECODE, dict(n_layers=65535), dict(n_layers=65536)),
    (EVICT, dict(H_kv=65535), dict(H_kv=65536)),
])
def test_the_documented_limits(op, at, beyond):
    assert status(op, **at) == 0
    assert status(op, **{**at, **beyond}) == 2
