"""Python binding of draft verification in include/cllm_verify.h (argument marshalling only).

After the target's logits of a step over blocks of drafted tokens::

    verifier = DraftVerifier(max_rows, max_batch)
    accepted, following = verifier.verify(logits, tokens, rows, uniforms=u, race=e, temperature=t)

``rows`` is the step's ``paged.PageRows``; what stands is committed (``paged.plan`` with
ctx + accepted gives the other tokens' pages back), and ``following`` begins the next block.
Conventions are those of ``paged``.
"""
from __future__ import annotations

import ctypes
import struct
from contextlib import nullcontext

import torch

from . import cllm as _c
from . import paged as _paged
from .paged import _INT_MAX, DTYPES, _stream, _Tensor, _vector

# Every function declared in include/cllm_verify.h.
EXPORTS = ("cllm_verifier_create", "cllm_verifier_destroy", "cllm_verify")

# cllm_verify_args as it lies in memory (native alignment).
_ARGS = struct.Struct("@4iPq6PqPq3P")
# What marshal.cpp keeps of a verifier: the call, the handle and the device.
_VERIFIER = struct.Struct("@2P2i")

_lib = None


def load():
    """The library with this header's signatures."""
    global _lib
    if _lib is None:
        lib = _paged.load()
        vp, i = ctypes.c_void_p, ctypes.c_int
        lib.cllm_verifier_create.argtypes = [i, i, ctypes.POINTER(vp)]
        lib.cllm_verifier_destroy.argtypes = [vp]
        lib.cllm_verifier_destroy.restype = None
        lib.cllm_verify.argtypes = [vp, vp, vp]
        lib.cllm_verifier_create.restype = lib.cllm_verify.restype = i
        _lib = lib
    return _lib


class DraftVerifier:
    """Scratch of verifications of up to max_rows rows and max_batch requests on a device."""

    def __init__(self, max_rows: int, max_batch: int, device="cuda"):
        lib = load()
        self.max_rows, self.max_batch = max_rows, max_batch
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device: need a CUDA device")
        if not all(-_INT_MAX <= x <= _INT_MAX for x in (max_rows, max_batch)):  # (ctypes would cut them to 32 bits)
            raise ValueError("max_rows, max_batch: at most 2^31 - 1")
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            self._dev = torch.cuda.current_device()
            _c._check(lib.cllm_verifier_create(max_rows, max_batch, ctypes.byref(h)), "cllm_verifier_create")
        self.device = torch.device("cuda", self._dev)
        self._h, self._lib = h, lib
        self._packed = _VERIFIER.pack(ctypes.cast(lib.cllm_verify, ctypes.c_void_p).value, h.value, self._dev, 0)
        self._verify = None if _paged._marshal is None else _paged._marshal.verify
        self._args = ctypes.create_string_buffer(_ARGS.size)
        self._argp = ctypes.addressof(self._args)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.cllm_verifier_destroy(self._h)
            self._h = self._verify = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t, what: str, dtype, rows: int, vocab: int):
        """Rows of a vocabulary's values: (address, row stride)."""
        if isinstance(t, _Tensor) and t.dtype is dtype and t.get_device() == self._dev and t.dim() == 2:
            n, width = t.shape
            row, one = t.stride()
            if n >= rows and width == vocab and (one == 1 or vocab == 1):
                return t.data_ptr(), row
        raise ValueError(f"{what}: need [{rows}][{vocab}] {dtype} on {self.device}, rows contiguous")

    def verify(self, logits, tokens, rows, uniforms=None, race=None, temperature=None, draft_probs=None, accepted=None,
               next_tokens=None, target_probs=None, stream=None):
        """Judge the drafts of a step: tokens (int32 [T]) of the requests of ``rows`` against logits
        [T][vocab] (float32, bfloat16 or float16, any row stride).  Returns int32 [batch] tensors
        (accepted, next): how many tokens of each request stand, its first among them, and
        the token that follows them (0 and -1 for a request without rows, or refused by its plan).
        uniforms (float32 [T], in [0, 1)) and race (float32 [batch][vocab], exponentially distributed):
        the random numbers; without both all requests are greedy.  temperature: float32 [batch] (None: 1; 0:
        greedy).  draft_probs: float32 [T][vocab], row i the distribution that token i + 1 was
        drawn from (None: the drafts are certain).  accepted, next_tokens: outputs to fill (None: allocated on
        the stream of the call); target_probs: float32 [T] to fill with the target's probability of each row's draft."""
        b, dev, f32, i32 = rows.batch, self._dev, torch.float32, torch.int32
        if rows._dev != dev:
            raise ValueError("rows: on another device than the verifier")
        st = _stream(stream, dev)
        if accepted is None or next_tokens is None:
            with nullcontext() if stream is None else torch.cuda.stream(stream):
                accepted = torch.empty(b, dtype=i32, device=self.device) if accepted is None else accepted
                next_tokens = torch.empty(b, dtype=i32, device=self.device) if next_tokens is None else next_tokens
        if self._verify is not None:
            rc = self._verify(self._packed, b, rows._start, rows._len, logits, tokens, uniforms, race, temperature, draft_probs,
                              accepted, next_tokens, target_probs, st)
            if rc is not None:
                if rc:
                    _c._check(rc, "cllm_verify")
                return accepted, next_tokens
        # (arguments that it does not take: looked at one by one)
        if not isinstance(logits, _Tensor) or logits.dim() != 2 or logits.dtype not in DTYPES:
            raise ValueError("logits: need a [rows][vocab] tensor of float32, bfloat16 or float16")
        t, vocab = logits.shape
        lp, ls = self._rows(logits, "logits", logits.dtype, t, vocab)
        tp = _vector(tokens, "tokens", i32, dev, t)
        up = rp = rs = hp = qp = qs = pp = 0
        if uniforms is not None:
            up = _vector(uniforms, "uniforms", f32, dev, t)
        if race is not None:
            rp, rs = self._rows(race, "race", f32, b, vocab)
        if temperature is not None:
            hp = _vector(temperature, "temperature", f32, dev, b)
        if draft_probs is not None:
            qp, qs = self._rows(draft_probs, "draft_probs", f32, t, vocab)
        ap = _vector(accepted, "accepted", i32, dev, b)
        np = _vector(next_tokens, "next_tokens", i32, dev, b)
        if target_probs is not None:
            pp = _vector(target_probs, "target_probs", f32, dev, t)
        _ARGS.pack_into(self._args, 0, b, t, vocab, DTYPES[logits.dtype], lp, ls, tp, rows._start, rows._len, hp, up, rp, rs, qp,
                        qs, ap, np, pp)
        rc = self._lib.cllm_verify(self._h, self._argp, st)
        if rc:
            _c._check(rc, "cllm_verify")
        return accepted, next_tokens
