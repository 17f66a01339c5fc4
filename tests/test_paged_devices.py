"""Which device a call of the paged cache runs on, and refusals of what lies on another, with
a stand-in for the library (CPU, no GPU)."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import paged


class Library:
    """Notes the device that is current when a call comes in."""

    def __init__(self):
        self.current, self.calls = 0, []

    def cllm_page_plan(self, *args):
        self.calls.append((self.current, args))
        return 0


@pytest.fixture
def lib(monkeypatch):
    lib = Library()

    @contextlib.contextmanager
    def device(index):
        before, lib.current = lib.current, index
        yield
        lib.current = before

    monkeypatch.setattr(paged, "load", lambda: lib)
    monkeypatch.setattr(paged, "_device", lambda: lib.current, raising=False)
    monkeypatch.setattr(paged, "_current", lambda index: 1000 + index)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(paged, "_tensor", lambda t, *a: t.data_ptr())
    return lib


def _tables(dev):
    t = object.__new__(paged.PageTables)
    t.__dict__.update(held=True, _dev=dev, _p=1)
    return t


def _rows(dev):
    r = object.__new__(paged.PageRows)
    r.__dict__.update(slots=True, _dev=dev, _p=2, _max=4)
    return r


LEN = torch.zeros(3, dtype=torch.int32)


@pytest.mark.parametrize("dev", [0, 1])
def test_a_plan_runs_on_its_tensors_device(lib, dev):
    paged.plan(_tables(dev), _rows(dev), LEN, LEN)
    assert [c for c, _ in lib.calls] == [dev]
    assert lib.calls[0][1][-1] == 1000 + dev
    assert lib.current == 0


@pytest.mark.parametrize("rows,out", [(0, 1), (1, 0), (0, 0)])
def test_a_plan_refuses_rows_and_tables_of_another_device(lib, rows, out):
    with pytest.raises(ValueError, match="device"):
        paged.plan(_tables(1), _rows(rows), LEN, LEN, out=_tables(out))
    assert not lib.calls


def test_a_stream_of_another_device_is_refused(lib):
    stream = types.SimpleNamespace(cuda_stream=5, device_index=0)
    with pytest.raises(ValueError, match="stream"):
        paged.plan(_tables(1), _rows(1), LEN, LEN, stream=stream)
    assert not lib.calls
    paged.plan(_tables(0), _rows(0), LEN, LEN, stream=stream)
    assert lib.calls[0][1][-1] == 5
