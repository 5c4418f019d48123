"""The binding's work memory for the operators, without a GPU: a library and streams that stand in for the
real ones note whose memory a call is given, and that it is held while it is used."""
import ctypes as C
import threading
import types
import weakref

import pytest
import torch

import paper_2607_05272_amd.sim as binding

CONTEXT, OTHER = 100, 200   # raw streams


class Stream:
    def __init__(self, raw, log):
        self.cuda_stream, self.log = raw, log

    def wait_stream(self, other):
        self.log.append(("wait", self.cuda_stream, other.cuda_stream))


@pytest.fixture
def world(monkeypatch):
    """A context on device 0 with the stream CONTEXT; what the tests change is in it."""
    w = types.SimpleNamespace(current=CONTEXT, device=0, capturing=set(), log=[], made=[], calls=[], need=64)
    w.streams = {r: Stream(r, w.log) for r in (CONTEXT, OTHER)}
    empty = torch.empty

    def make(n, dtype, device):
        t = empty(n, dtype=dtype)
        w.made.append(weakref.ref(t))
        return t

    def op_work(sizes, out):
        out._obj.value = w.need
        return 0

    def op(ctx, sizes, *args):
        held = [r() for r in w.made]
        w.calls.append(types.SimpleNamespace(at=args[-2], bytes=args[-1], held=[t is not None and t.data_ptr() == args[-2]
                                                                               for t in held]))
        w.log.append(("call", args[-2]))
        return 0
    monkeypatch.setattr(binding.torch, "empty", make)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: w.current, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: w.device)
    # as torch has it: of the current device's stream
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: w.device in w.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: w.streams[w.current])
    s = object.__new__(binding.Sim)
    s.lib = types.SimpleNamespace(op=op, op_work=op_work)
    s._ctx, s._index, s._device = None, 0, torch.device("cuda", 0)
    s._raw_stream, s.stream, s._work = CONTEXT, w.streams[CONTEXT], threading.local()
    w.sim = s
    w.call = lambda: s._call("op", C.c_int(0)) or w.calls[-1]
    return w


def test_calls_on_the_contexts_stream_share_a_threads_memory(world):
    a, b = world.call(), world.call()
    assert a.at == b.at and b.bytes == 64 and any(b.held)
    assert not any(l[0] == "wait" for l in world.log)
    world.need = 128
    c = world.call()
    assert c.bytes == 128 and any(c.held)
    other = []
    t = threading.Thread(target=lambda: other.append(world.call()))
    t.start()
    t.join()
    assert other[0].at != c.at and any(other[0].held)
    world.need = 0
    d = world.call()
    assert d.at is None and d.bytes == 0


def test_memory_of_a_call_from_another_stream_is_held_until_that_stream_waits(world):
    """Until then another thread's allocation on that stream could be given the same bytes, and nothing would
    order its work after this call's."""
    kept = world.call().at
    world.log.clear()
    world.current = OTHER
    c = world.call()
    assert c.at != kept and any(c.held)
    assert world.log == [("wait", CONTEXT, OTHER), ("call", c.at), ("wait", OTHER, CONTEXT)]
    assert world.made[-1]() is None          # and no longer


def test_captured_calls_have_memory_of_their_own(world):
    kept = world.call().at
    world.capturing = {0}
    c = world.call()
    assert c.at != kept and any(c.held)
    world.capturing = set()
    assert world.call().at == kept


def test_another_current_device_takes_memory_of_its_own(world):
    """Whether the context's stream is being captured can be asked only of the current device's: a call made
    while that is another one does not use the memory that eager calls share."""
    kept = world.call().at
    world.capturing, world.device = {0}, 1
    c = world.call()
    assert c.at != kept and any(c.held)
    world.capturing, world.device = set(), 0
    assert world.call().at == kept
