"""Streams that the operators' Python calls are given, without a GPU: stand-ins for tensors and streams."""
import pytest
import torch

import paper_2607_18957_gb300 as cfa
from paper_2607_18957_gb300 import build as cfa_build
from paper_2607_18957_gb300 import ops


class OnDevice1:
    """What the calls ask of an operand before they enter the stream's guard."""
    requires_grad = False
    device = torch.device("cuda", 1)

    def get_device(self):
        return 1


class Entered(Exception):
    """Far enough: the call has entered the guard."""


class Stream:
    def __init__(self, index):
        self.device = torch.device("cuda", index)


@pytest.fixture(autouse=True)
def started(monkeypatch):
    cfa_build.build()
    if ops.torch is None:
        ops._start()
    entered = []

    class Guard:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream)
            raise Entered

        def __exit__(self, *exc):
            pass

    monkeypatch.setattr(torch.cuda, "stream", Guard)
    monkeypatch.setattr(ops, "_device", lambda: 0)
    return entered


CALLS = [lambda x, s: cfa.linear(x, x, stream=s), lambda x, s: cfa.route(x, 2, stream=s),
         lambda x, s: cfa.experts(x, x, x, x, x, stream=s)]


@pytest.mark.parametrize("call", CALLS, ids=["linear", "route", "experts"])
def test_a_stream_of_another_device_is_refused(call, started):
    with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
        call(OnDevice1(), Stream(0))
    assert started == []


@pytest.mark.parametrize("call", CALLS, ids=["linear", "route", "experts"])
def test_a_stream_of_the_operands_device_is_entered(call, started):
    s = Stream(1)
    with pytest.raises(Entered):
        call(OnDevice1(), s)
    assert started == [s]
