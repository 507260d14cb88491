"""A decoding step's operators at the edges of what their documentation allows (no GPU)."""
import math

import pytest
import torch

import paper_2607_18957_gb300 as cfa
from paper_2607_18957_gb300 import build as cfa_build
from paper_2607_18957_gb300 import ops, step


@pytest.mark.parametrize("dim,base,length,factor", [
    (128, 10000.0, 131072, 4.0), (128, 10000.0, 131072, 8.0), (128, 10000.0, 65536, 8.0),
    (64, 10000.0, 65536, 4.0), (64, 10000.0, 131072, 4.0), (64, 10000.0, 163840, 16.0),
    (128, 10000.0, 4096, 16.0), (64, 1e6, 32768, 4.0), (2, 10000.0, 131072, 2.0)])
def test_ramp_goes_on_behind_the_last_pair(dim, base, length, factor):
    """Pair by pair, with the ramp's ends found by counting turns instead of by logarithms: the index
    (of a pair or behind the last) from which on all turn fewer than 32 times, less one, and the first
    that turns no more than once."""
    def turns(i):
        return length * base ** (-2 * i / dim) / (2 * math.pi)
    first = next(i for i in range(10 * dim) if turns(i + 1) < 32)
    last = next(i for i in range(10 * dim) if turns(i) <= 1)
    f, _ = cfa.rotary_frequencies(dim, base, scaling="ramp", factor=factor, length=length)
    assert len(f) == dim // 2
    for i, v in enumerate(f):
        g = base ** (-2 * i / dim)
        share = min(max((i - first) / (last - first), 0.0), 1.0)  # of the frequency that is divided
        assert v == pytest.approx(g * (1 - share) + g / factor * share, rel=1e-12, abs=0.0), i


def test_ramp_leaves_pairs_that_turn_often_alone():
    """128 values, base 10000, 131,072 positions: 32 turns at index 45.03, one at 69.1, so that the last
    pair, 63, keeps 7 / 25 of its frequency and an eighth of the rest."""
    f, _ = cfa.rotary_frequencies(128, 10000.0, scaling="ramp", factor=8.0, length=131072)
    assert f[45] == pytest.approx(10000.0 ** (-45 / 64), rel=1e-12, abs=0.0)
    assert f[63] == pytest.approx(10000.0 ** (-63 / 64) * (7 / 25 + 18 / 25 / 8), rel=1e-12, abs=0.0)


@pytest.mark.parametrize("low,high", [(1.0, 1.0), (4.0, 1.0), (1.0, math.nan)])
def test_bands_that_are_none_are_refused(low, high):
    """Between low and high turns the frequencies pass over: the other way round they would be divided
    where they are to be kept."""
    with pytest.raises(ValueError, match="low .*high"):
        cfa.rotary_frequencies(64, scaling="bands", factor=2.0, length=4096, low=low, high=high)


class FakeStream:
    """torch's current stream: a foreign one's id is its handle."""
    device = "somewhere"

    def __init__(self, id, log):
        self.stream_id, self.log = id, log

    def wait_event(self, event):
        self.log.append(("waits", self.stream_id, event.number))


def test_a_foreign_handle_may_name_another_stream_by_now(monkeypatch):
    """Its kept workspace is used by a call that waits for the one before; torch's own streams need no
    waits, and an old foreign one's memory goes back only behind its last call."""
    cfa_build.build()
    if ops.torch is None:
        ops._start()
    log, current = [], []

    class Event:
        made = 0

        def __init__(self):
            self.number = Event.made
            Event.made += 1

    class Memory:
        def __init__(self, need, **kw):
            self.need = need

        def numel(self):
            return self.need

        def record_stream(self, stream):
            log.append(("kept for", stream.stream_id, self.need))

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: current[-1])
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch, "empty", Memory)
    monkeypatch.setattr(step, "_KEPT", {})
    monkeypatch.setattr(step, "_FOREIGN", {})

    def call(handle, need, id=None):
        current.append(FakeStream(handle if id is None else id, log))
        return step._kept(0, handle, need)
    a, last = call(0x1000, 10)
    assert last.number == 0 and log == []
    b, again = call(0x1000, 10)
    assert b is a and again is last and log == [("waits", 0x1000, 0)]
    c, again = call(0x1000, 20)  # a larger one, behind the call with the smaller
    assert c is not a and c.need == 20 and again is last and log == 2 * [("waits", 0x1000, 0)]
    assert step._KEPT == {}
    del log[:]
    for handle, id in ((0, 0), (0x2000, 35)):  # torch's default stream and one of its pool
        w, last = call(handle, 10, id)
        assert last is None and step._KEPT[0, handle] is w
    for i in range(64):
        call(0x10000 + 16 * i, 1)
    assert log == [("waits", 0x10000 + 16 * 63, 0), ("kept for", 0x10000 + 16 * 63, 20)]
    assert len(step._FOREIGN) == 64 and (0, 0x1000) not in step._FOREIGN


P, MIB, INVAL = 0x7F0000000000, 1 << 20, -1


@pytest.mark.parametrize("scale", [2.3e38, 2.4e38, 3.4e38])
def test_logprobs_scale_has_room_in_powers_of_two(scale):
    """The kernel's exponents are of 2: scale * log2(e) is finite, or the call is refused."""
    lib = _library()
    args = step._LOGPROBS.pack(P, P + 8 * MIB, P + 9 * MIB, P + 10 * MIB, 0, 0, 0, 100, 100,
                               cfa._lib.DTYPE["f32"], 0, scale, 0)
    assert lib.cfa_logprobs_async(args, None) == (0 if scale < 2.35e38 else INVAL)


@pytest.mark.parametrize("scale,k_scale,ok", [(2.3e38, 1.0, True), (-2.4e38, 1.0, False), (1e30, 1e9, False),
                                              (1e20, 1e17, True), (3e38, 0.1, False)])
def test_attend_scales_have_room_in_powers_of_two(scale, k_scale, ok):
    """scale * log2(e), and that times the keys' scale."""
    lib = _library()
    f8 = step.F8_E4M3 if k_scale != 1.0 else cfa._lib.DTYPE["bf16"]
    args = step._ATTEND.pack(P, P + 8 * MIB, P + 16 * MIB, P + MIB, P + 2 * MIB, P + 3 * MIB, 0, P + 64 * MIB,
                             64 * MIB, 0, 256, 256, 4, 2048, 128, 64, 2048, 128, 64, 1, 4, 8, 16, 4, 2, 64, 0,
                             cfa._lib.DTYPE["bf16"], f8, 0, scale, k_scale, 1.0)
    assert lib.cfa_attend_async(args, None) == (0 if ok else INVAL)


def _library():
    cfa_build.build()
    return cfa._lib.load()
