"""Rotary frequencies and the refusals of the table call and of writes with norms (CPU, no GPU: only
invalid calls are made)."""
import ctypes
import math
from array import array

import pytest

from paper_2403_00835_gb300 import cllm, paged

EINVAL, EUNSUPPORTED = -1, -8
P = 0x1000  # never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    return paged.load()


def test_frequencies_by_hand():
    assert list(paged.rope_frequencies(4, 1e4)) == [1.0, 1e-2]
    assert list(paged.rope_frequencies(4, 1e4, "linear", 8.0)) == [0.125, 1e-2 / 8]
    base = paged.rope_frequencies(8, 1e4, "base", 4.0)
    assert base[0] == 1.0 and base[3] == pytest.approx(1e4 ** (-6 / 8) / 4.0, rel=1e-14)
    # 1000 positions are 159 turns of the first pair (kept), 15.9 of the second (a mix), 0.159 of the last (divided)
    f = paged.rope_frequencies(6, 1e3, "ramp", 4.0, trained=1000)
    t = 1000 * 0.1 / (2 * math.pi)
    keep = (t - 1.0) / 31.0
    assert list(f) == pytest.approx([1.0, 0.1 * keep + 0.025 * (1 - keep), 0.01 * ((1000 * 0.01 / (2 * math.pi) - 1) / 31)
                                     + 0.0025 * (1 - (1000 * 0.01 / (2 * math.pi) - 1) / 31)], rel=1e-14)


@pytest.mark.parametrize("a", [(3,), (0,), (-2,), (8, 0.0), (8, math.nan), (8, 1e4, "other"), (8, 1e4, "linear", 0.0),
                               (8, 1e4, "linear", math.inf), (2, 1e4, "base", 2.0), (8, 1e4, "ramp", 2.0),
                               (8, 1e4, "ramp", 2.0, 100, 1.0, 1.0)])
def test_frequencies_refuse(a):
    with pytest.raises(ValueError):
        paged.rope_frequencies(*a)


def _table(lib, table=P, first=0, positions=4, dims=4, f=(1.0, 0.5), amplitude=1.0):
    f = array("d", f) if f is not None else None
    return lib.cllm_rope_table(table, first, positions, dims, None if f is None else f.buffer_info()[0], amplitude, None)


@pytest.mark.parametrize("kw", [dict(table=None), dict(table=P + 8), dict(first=-1), dict(positions=-1),
                                dict(first=2 ** 31 - 4), dict(dims=0), dict(dims=3), dict(dims=258), dict(f=None),
                                dict(f=(1.0, math.nan)), dict(f=(math.inf, 1.0)), dict(f=(-2.0 ** 21, 1.0)),
                                dict(amplitude=math.inf), dict(amplitude=math.nan)])
def test_table_refuses(lib, kw):
    assert _table(lib, **kw) == EINVAL


def test_a_table_of_no_positions_is_nothing_to_do(lib):
    assert _table(lib, positions=0) == 0


def test_a_host_table_is_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="CUDA"):
        paged.rope_table(4, [1.0], out=torch.zeros(4, 1, 2))


@pytest.mark.parametrize("positions,first", [(-1, 0), (2 ** 32 + 4, 0), (4, 2 ** 32), (4, -2), (4, 2 ** 31 - 3), (2 ** 31, 0)])
def test_positions_past_31_bits_are_refused(positions, first):
    """(Not cut to the bits that the library takes.)"""
    with pytest.raises(ValueError, match="positions"):
        paged.rope_table(positions, [1.0], first=first)


def test_null_handles(lib):
    zeros = ctypes.create_string_buffer(256)
    at = ctypes.addressof(zeros)
    assert lib.cllm_paged_append_heads(None, at, at, None) == EINVAL
    assert lib.cllm_paged_append_heads(at, at, None, None) == EINVAL


def test_the_packed_arguments_are_where_the_library_reads_them():
    class Rows(ctypes.Structure):
        _fields_ = [("layer", ctypes.c_int), ("rows", ctypes.c_int), *[(n, ctypes.c_void_p) for n in "kvqo"],
                    *[(n, ctypes.c_int64) for n in ("ks", "vs", "qs", "os")], *[(n, ctypes.c_void_p) for n in ("slots", "rope", "pos")],
                    ("max_pos", ctypes.c_int)]

    class Heads(ctypes.Structure):
        _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("eps", ctypes.c_float), ("dims", ctypes.c_int),
                    ("interleaved", ctypes.c_int)]

    assert ctypes.sizeof(Rows) == paged._HEADS_AT and paged._HEADS_AT % ctypes.alignment(Heads) == 0
    buf = ctypes.create_string_buffer(paged._HEADS_AT + 64)
    paged._HEADS.pack_into(buf, paged._HEADS_AT, 5, 6, 0.5, 32, True)
    h = Heads.from_buffer(buf, paged._HEADS_AT)
    assert (h.q, h.k, h.eps, h.dims, h.interleaved) == (5, 6, 0.5, 32, 1)
    assert cllm.STATUS[EUNSUPPORTED] == "CLLM_EUNSUPPORTED"


def test_a_null_cache_with_first_tokens(lib):
    zeros = ctypes.create_string_buffer(256)
    assert lib.cllm_paged_attention_sinks(None, ctypes.addressof(zeros), 4, None) == EINVAL


@pytest.mark.parametrize("dev", [0, 1])
def test_a_table_is_filled_on_its_device(dev, monkeypatch):
    """With a stand-in for the library, which notes the device that is current."""
    import contextlib
    import types
    torch = pytest.importorskip("torch")
    current, calls = [0], []

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    def call(*args):
        calls.append((current[0], args))
        return 0

    monkeypatch.setattr(paged, "_lib", types.SimpleNamespace(cllm_rope_table=call))
    monkeypatch.setattr(paged, "_device", lambda: current[0])
    monkeypatch.setattr(paged, "_current", lambda index: 1000 + index)
    monkeypatch.setattr(paged, "_tensor", lambda t, *a: 64)
    monkeypatch.setattr(torch.cuda, "device", device)
    out = types.SimpleNamespace(get_device=lambda: dev)
    assert paged.rope_table(4, [1.0, 0.5], out=out) is out
    assert [(c, a[0], a[1:4], a[-1]) for c, a in calls] == [(dev, 64, (0, 4, 4), 1000 + dev)] and current == [0]
    with pytest.raises(ValueError, match="stream"):
        paged.rope_table(4, [1.0, 0.5], out=out, stream=types.SimpleNamespace(cuda_stream=5, device_index=1 - dev))
    assert len(calls) == 1
