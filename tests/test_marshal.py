"""The native look at a call's tensors (CPU, no GPU): what it does not take it hands back, and nothing is called."""
import struct

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged, verify

P = 0x1000  # never called or dereferenced: the checks fail first


@pytest.fixture(scope="module")
def native():
    paged.load()
    if paged._marshal is None:
        pytest.skip("not built here")
    return paged._marshal


def test_numbers_of_arguments(native):
    for f, n in ((native.append, 14), (native.attention, 15), (native.rope_table, 8), (native.verify, 14)):
        assert f() is None
        assert f(*[None] * n) is None
        assert f(*[None] * (n + 1)) is None


def test_host_tensors_are_not_taken(native):
    cache = paged._CACHE.pack(P, P, P, P, 0, 0, 64, 2, 4, 0)
    k, slots = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int64)
    assert native.append(cache, 0, k, k, slots, None, None, None, None, None, None, 1e-6, False, 0) is None
    assert native.append(cache[:-4], 0, k, k, slots, None, None, None, None, None, None, 1e-6, False, 0) is None
    assert native.attention(cache, 0, k, k, None, P, P, 1, P, 4, 1.0, 0, 0, None, 0) is None
    assert native.rope_table(P, 3, [1.0], 1.0, 0, torch.zeros(3, 1, 2), 0, 0) is None
    v = verify._VERIFIER.pack(P, P, 0, 0)
    z, i = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    assert native.verify(v, 1, P, P, z, i, None, None, None, None, i, i, None, 0) is None


@pytest.mark.parametrize("bad", [2 ** 40, -1, 1.5, None, "0"])
def test_numbers_that_the_library_does_not_take(native, bad):
    cache = paged._CACHE.pack(P, P, P, P, 0, 0, 64, 2, 4, 0)
    k, slots = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int64)
    assert native.append(cache, bad, k, k, slots, None, None, None, None, None, None, 1e-6, False, 0) is None
    assert native.attention(cache, 0, k, k, None, P, P, 1, P, 4, 1.0, bad, 0, None, 0) is None
    assert native.rope_table(P, bad, [1.0], 1.0, 0, k, 0, 0) is None


def test_what_is_kept_of_a_handle_is_what_the_library_reads():
    assert paged._CACHE.size == struct.calcsize("@4P6i") == 56 and verify._VERIFIER.size == 24
