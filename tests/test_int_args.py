"""Numbers past 31 bits on either side, which would reach the library as others (CPU, no GPU)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged, verify

FAR = [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32 + 5, -2 ** 64 + 5]


@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("which", [0, 1])
def test_a_verifiers_sizes(far, which):
    with pytest.raises(ValueError, match="at most"):
        verify.DraftVerifier(*((far, 5) if which == 0 else (5, far)))


@pytest.mark.parametrize("far", FAR)
def test_first_tokens(far):
    cache = object.__new__(paged.PagedCache)
    cache.__dict__.update(_dev=0, dtype=torch.float32, _h=None)
    q = torch.zeros(1, 4, 64)
    rows, tables = object.__new__(paged.PageRows), object.__new__(paged.PageTables)
    with pytest.raises(ValueError, match="sinks"):
        cache.attention(0, q, rows, tables, out=q, window=4, sinks=far)
