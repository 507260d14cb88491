"""Streams that the operators' calls are given as handles, without a GPU: stand-ins for torch's streams."""
import itertools
import threading

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

    numbers = itertools.count()
    monkeypatch.setattr(torch.cuda, "Stream", lambda device: Stream(f"own {next(numbers)} on {device}"))
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: Stream(f"default on {device}"))
    monkeypatch.setattr(torch.cuda, "stream", Guard)
    return done


@pytest.mark.parametrize("handle,name", [(0, "default on 3"), (1, "default on 3"), (4096, "4096 on 3"),
                                         (-1, "-1 on 3")])
def test_handles_name_their_streams(log, handle, name):
    """0 and cudaStreamLegacy are the default stream."""
    with ops._elsewhere(handle, 3):
        log.append("call")
    assert log == [("enter", name), "call", ("exit", name)]


def test_every_thread_has_a_stream_in_the_place_of_the_handle_that_names_its_own(log):
    """cudaStreamPerThread, 2, is another stream in every thread: calls go to a stream of the thread's,
    between what is before and behind them on that of the handle."""
    def work(devices):
        for d in devices:
            with pytest.raises(KeyError):
                with ops._elsewhere(2, d):
                    log.append("call")
                    raise KeyError  # a refusal leaves the streams joined too
    for devices in ((0, 0, 1), (0,)):
        t = threading.Thread(target=work, args=(devices,))
        t.start()
        t.join()
    want = []
    for own, d in ((0, 0), (0, 0), (1, 1), (2, 0)):
        own, theirs = f"own {own} on {d}", f"2 on {d}"
        want += [(own, "waits for", theirs), ("enter", own), "call", ("exit", own),
                 (theirs, "waits for", own)]
    assert log == want
