"""The native look at a call's numbers: with tensors that are all right, a number outside its range or of another type is handed
back and nothing is called; one inside it reaches the call (a stand-in that notes what it gets)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import cllm, paged, verify

pytestmark = pytest.mark.gpu

P, I = ctypes.c_void_p, ctypes.c_int
WRONG = [2 ** 31, 2 ** 32 + 1, 2 ** 40, 2 ** 70, -1, -2 ** 32 + 1, -2 ** 70, 1.0, None, "1", True]


class StandIn:
    """Calls of three pointers (append's have a fourth kind), and of a rotary table."""

    def __init__(self):
        self.got = []
        self.three = ctypes.CFUNCTYPE(I, P, P, P)(lambda h, args, s: self.note("three", h, args, s))
        self.heads = ctypes.CFUNCTYPE(I, P, P, P, P)(lambda h, args, heads, s: self.note("heads", h, args, s))
        self.sinks = ctypes.CFUNCTYPE(I, P, P, I, P)(lambda h, args, n, s: self.note("sinks", h, args, s, n))
        self.rope = ctypes.CFUNCTYPE(I, P, I, I, I, P, ctypes.c_float, P)(self.note_rope)

    def note(self, kind, handle, args, stream, *more):
        self.got.append((kind, handle, (I * 4).from_address(args)[:], stream, *more))
        return 7

    def note_rope(self, out, first, positions, dims, f, amplitude, stream):
        self.got.append(("rope", first, positions, dims, (ctypes.c_double * (dims // 2)).from_address(f)[:], amplitude, stream))
        return 7

    def taken(self, rc):
        """What the call got, which is all of it and answered 7."""
        assert rc == 7 and len(self.got) == 1
        return self.got.pop()

    def handed_back(self, rc):
        assert rc is None and not self.got


@pytest.fixture
def native():
    paged.load()
    if paged._marshal is None:
        pytest.skip("not built here")
    return paged._marshal


@pytest.fixture
def lib():
    return StandIn()


def _at(f):
    return ctypes.cast(f, P).value


def _cache(lib):
    return paged._CACHE.pack(_at(lib.three), _at(lib.heads), _at(lib.sinks), 0x50, cllm.CLLM_F32, 0, 64, 2, 4, 0)


def _append(lib):
    k = torch.zeros(3, 2, 64, device="cuda")
    q, slots = torch.zeros(3, 4, 64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    rope, pos = torch.zeros(9, 16, 2, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    return [_cache(lib), 5, k, k, slots, q, None, rope, pos, None, torch.zeros(64, device="cuda"), 1e-6, False, 0x60]


def test_append(native, lib):
    ok = _append(lib)
    kind, handle, (layer, rows, *_), stream = lib.taken(native.append(*ok))
    assert (kind, handle, layer, rows, stream) == ("heads", 0x50, 5, 3, 0x60)
    assert lib.taken(native.append(*ok[:1], 2 ** 31 - 1, *ok[2:]))[2][0] == 2 ** 31 - 1
    plain = ok[:5] + [None] * 6 + ok[11:]
    assert lib.taken(native.append(*plain))[0] == "three"
    for bad in WRONG:
        lib.handed_back(native.append(*ok[:1], bad, *ok[2:]))
    for at, values in ((11, (1, None, "0")), (12, (0, 1, None)), (13, (1.0, None, True)), (0, (ok[0][:-4], ok[0] + b"\0" * 4, None, 3))):
        for bad in values:
            lib.handed_back(native.append(*ok[:at], bad, *ok[at + 1:]))
    lib.handed_back(native.append(*ok[:-1]))
    lib.handed_back(native.append(*ok, 0))


def test_append_tensors(native, lib):
    ok = _append(lib)
    wide = torch.zeros(3, 8, 128, device="cuda")
    for at, values in ((2, (wide[:, :2, :64], wide[:, ::2, :64][:, :2], ok[2].half(), ok[2][:2], ok[2].cpu(), None)),
                       (3, (ok[3][:2], ok[3].double())), (4, (ok[4][:2], ok[4].int(), ok[4].cpu())), (5, (ok[2], ok[5][:2])),
                       (6, (ok[2], ok[5].half())), (7, (ok[7][..., :1], ok[7].double(), ok[7][:, ::2], torch.zeros(9, 33, 2, device="cuda"))),
                       (8, (ok[8][:2], ok[8].long(), None)), (9, (ok[10][:32], ok[10].half())), (10, (ok[10].view(8, 8),))):
        for bad in values:
            lib.handed_back(native.append(*ok[:at], bad, *ok[at + 1:]))


def test_attention(native, lib):
    q = torch.zeros(3, 4, 64, device="cuda")
    ok = [_cache(lib), 5, q, torch.zeros_like(q), None, 0x10, 0x20, 6, 0x30, 9, 1.0, 11, 12, None, 0x60]
    kind, handle, (layer, batch, rows, _), stream, sinks = lib.taken(native.attention(*ok))
    assert (kind, handle, layer, batch, rows, stream, sinks) == ("sinks", 0x50, 5, 6, 3, 0x60, 12)
    assert lib.taken(native.attention(*ok[:12], 2 ** 31 - 1, *ok[13:]))[4] == 2 ** 31 - 1
    for at in (1, 7, 9, 11, 12):
        for bad in WRONG:
            lib.handed_back(native.attention(*ok[:at], bad, *ok[at + 1:]))
    for at, values in ((10, (1, None)), (5, (None, 1.0)), (14, (None, True)), (0, (ok[0][:-4],)), (2, (q[:2], q[:, :3], q.half())),
                       (4, (torch.zeros(3, 3, device="cuda"), torch.zeros(3, 4, device="cuda").half())),
                       (13, (torch.zeros(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda")))):
        for bad in values:
            lib.handed_back(native.attention(*ok[:at], bad, *ok[at + 1:]))


def test_rope_table(native, lib):
    out = torch.zeros(4, 3, 2, device="cuda")
    ok = [_at(lib.rope), 4, [1.0, 2.0, 3.0], 0.5, 9, out, 0, 0x60]
    assert lib.taken(native.rope_table(*ok)) == ("rope", 9, 4, 6, [1.0, 2.0, 3.0], 0.5, 0x60)
    assert lib.taken(native.rope_table(*ok[:4], 2 ** 31 - 5, *ok[5:]))[1] == 2 ** 31 - 5
    for at in (1, 4):
        for bad in WRONG + [2 ** 31 - 4]:  # (with the others past 2^31 - 1 in all)
            lib.handed_back(native.rope_table(*ok[:at], bad, *ok[at + 1:]))
    for at, values in ((2, ([1.0, 2.0], [1.0, 2.0, 3], (1.0, 2.0, 3.0), None, [])), (3, (1, None)), (5, (out[:3], out[..., :1], out.half(), out.cpu())),
                       (6, (1, 2 ** 40, None)), (7, (None, 1.0))):
        for bad in values:
            lib.handed_back(native.rope_table(*ok[:at], bad, *ok[at + 1:]))


def test_verify(native, lib):
    v = verify._VERIFIER.pack(_at(lib.three), 0x50, 0, 0)
    z, i, f = torch.zeros(5, 8, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")
    race = torch.zeros(2, 8, device="cuda")
    ok = [v, 2, 0x10, 0x20, z, i, f, race, f[:2], z, i, i, f, 0x60]
    assert lib.taken(native.verify(*ok)) == ("three", 0x50, [2, 5, 8, cllm.CLLM_F32], 0x60)
    for bad in WRONG + [3]:  # (3: more requests than the race has rows)
        lib.handed_back(native.verify(*ok[:1], bad, *ok[2:]))
    for at, values in ((0, (v[:-4],)), (2, (None, 1.0)), (4, (z.double(), z[0], z.T, z.cpu(), None)), (5, (i[:4], i.long(), None)), (6, (f[:4],)),
                       (7, (race[:, :7], race.half())), (8, (f[:1],)), (9, (race,)), (10, (i[:1], None)), (11, (f,)), (12, (f[:4],)), (13, (None,))):
        for bad in values:
            lib.handed_back(native.verify(*ok[:at], bad, *ok[at + 1:]))
