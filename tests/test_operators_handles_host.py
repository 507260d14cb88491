"""Streams that the operators' calls are given as handles, without a GPU: stand-ins for torch's streams."""
import pytest
import torch

from paper_2607_18957_gb300 import build as cfa_build
from paper_2607_18957_gb300 import ops


@pytest.fixture
def log(monkeypatch):
    """What happens to the streams, in order."""
    cfa_build.build()
    if ops.torch is None:
        ops._start()
    done = []

    class Stream:
        def __init__(self, name):
            self.name = name

        def wait_stream(self, other):
            done.append((self.name, "waits for", other.name))

    class Guard:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            done.append(("enter", self.stream.name))

        def __exit__(self, *exc):
            done.append(("exit", self.stream.name))

    def external(handle, device=None):
        # what torch does: no stream at handle 0 is a request for one of its pool's, 1 is not known
        if handle == 0:
            return Stream("any of the pool")
        if handle == 1:
            raise RuntimeError("invalid StreamId1")
        return Stream(f"{handle} on {device}")

    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: Stream(f"default on {device}"))
    monkeypatch.setattr(torch.cuda, "stream", Guard)
    return done


@pytest.mark.parametrize("handle,name", [(0, "default on 3"), (1, "default on 3"), (4096, "4096 on 3")])
def test_handles_name_their_streams(log, handle, name):
    """0 and cudaStreamLegacy are the default stream."""
    with ops._elsewhere(handle, 3):
        log.append("call")
    assert log == [("enter", name), "call", ("exit", name)]
