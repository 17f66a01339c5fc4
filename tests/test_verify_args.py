"""Draft verification's refusals that need no GPU, and the tests' own model of it on hand-worked steps."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_2403_00835_gb300 import verify
from tests.test_abi import declared_functions
from tests.verify_util import Model

EINVAL = -1
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_00835_gb300", "csrc")


@pytest.fixture(scope="module")
def lib():
    return verify.load()


def test_every_call_is_bound_and_exported(lib):
    assert set(verify.EXPORTS) <= set(declared_functions())
    assert all(hasattr(lib, n) for n in verify.EXPORTS)


@pytest.mark.parametrize("rows,batch", [(0, 1), (-1, 1), (1, 0), (1, 4097), (2 ** 30 + 1, 1)])
def test_create_refuses(lib, rows, batch):
    h = ctypes.c_void_p()
    assert lib.cllm_verifier_create(rows, batch, ctypes.byref(h)) == EINVAL
    assert not h.value
    assert lib.cllm_verifier_create(4, 4, None) == EINVAL


def test_null_verifiers(lib):
    lib.cllm_verifier_destroy(None)  # no-op
    zeros = ctypes.create_string_buffer(256)
    assert lib.cllm_verify(None, ctypes.addressof(zeros), None) == EINVAL
    with pytest.raises(ValueError, match="device"):
        verify.DraftVerifier(4, 4, device="cpu")


@pytest.mark.parametrize("rows,batch", [(2 ** 32 + 1, 1), (1, 2 ** 32 + 1)])
def test_sizes_past_31_bits_are_refused(rows, batch):
    with pytest.raises(ValueError, match="at most"):
        verify.DraftVerifier(rows, batch)


def test_kernels_wait_before_they_read_with_coherent_loads():
    """They may start while the kernel before them is still writing what they read."""
    with open(os.path.join(CSRC, "verify.cu")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"__ldg\b|__restrict|ld\.global\.(\w+\.)*nc\b", code)
    kernels = code.split("__global__")[1:]
    assert len(kernels) == 2 and all("pdl_wait();" in k for k in kernels)


def test_the_packed_arguments_are_where_the_library_reads_them():
    P, Q, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int

    class Args(ctypes.Structure):
        _fields_ = [("batch", I), ("rows", I), ("vocab", I), ("dtype", I), ("logits", P), ("ls", Q), ("tokens", P), ("row_start", P),
                    ("seq_len", P), ("temperature", P), ("uniforms", P), ("race", P), ("rs", Q), ("probs", P), ("ps", Q),
                    ("accepted", P), ("next", P), ("target", P)]

    assert ctypes.sizeof(Args) == verify._ARGS.size
    buf = ctypes.create_string_buffer(verify._ARGS.size)
    verify._ARGS.pack_into(buf, 0, *range(1, 19))
    a = Args.from_buffer(buf)
    assert [getattr(a, f) for f, _ in Args._fields_] == list(range(1, 19))


def test_model_on_hand_worked_steps():
    p = np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1], [0.2, 0.2, 0.6]])
    z, race = np.log(p), np.array([1.0, 1.0, 1.0])
    # certain drafts: 0 stands below 0.5, 1 below 0.8; the last row's largest is 2
    m = Model(z, [7, 0, 1], race, [0.4, 0.7, 0.0])
    assert (m.accepted, m.next) == (3, 2) and np.allclose(m.probs, [0.5, 0.8, 0.0])
    # the first falls: of what is left 1 and 2 are alike, the race decides, then the lowest index
    assert (Model(z, [7, 0, 1], race, [0.5, 0.7, 0.0]).accepted, Model(z, [7, 0, 1], race, [0.6, 0.7, 0.0]).next) == (1, 1)
    assert Model(z, [7, 0, 1], np.array([1.0, 2.0, 1.0]), [0.6, 0.7, 0.0]).next == 2
    # a draft model's distribution: it stands below p / q; the rest is max(p - q, 0) = (0, 0.05, 0.15)
    q = np.array([[0.8, 0.2, 0.1], [1 / 3] * 3, [1 / 3] * 3])
    assert Model(z, [7, 0, 1], race, [0.62, 0.0, 0.0], q=q).accepted == 3
    m = Model(z, [7, 0, 1], race, [0.63, 0.0, 0.0], q=q)
    assert (m.accepted, m.next) == (1, 2)
    # a draft that is none; greedy; nothing to draw
    assert (Model(z, [7, -1, 1], race, [0.0] * 3).accepted, Model(z, [7, 3, 1], race, [0.0] * 3).next) == (1, 0)
    assert (Model(z, [7, 0, 0], race, [0.9] * 3, heat=0.0).accepted, Model(z, [7, 0, 0], race, [0.9] * 3, heat=0.0).next) == (2, 1)
    m = Model(np.full((1, 3), -np.inf), [7], race, [0.0])
    assert (m.accepted, m.next) == (1, -1)
