"""The order of calls that share an optimizer's table, on streams that are fakes: who waits for whom."""
import pytest
import torch


class Stream:
    def __init__(self, name, log):
        self.name, self.log, self.capturing, self.cuda_stream = name, log, False, id(self)

    def wait_stream(self, other):
        self.log.append((self.name, other.name))


class Tensor:
    def __init__(self):
        self.used = []

    def record_stream(self, stream):
        self.used.append(stream.name)


@pytest.fixture
def fake(monkeypatch):
    from paper_2407_17029_b200 import build
    build.build()
    from paper_2407_17029_b200 import binding as qb
    log = []
    streams = {n: Stream(n, log) for n in "abc"}
    monkeypatch.setattr(qb, "_capturing", lambda s: s.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: streams["a"])
    monkeypatch.setattr(qb, "_stream_ptr", lambda s: (s or streams["a"]).cuda_stream)
    t = Tensor()
    return qb._Order([t]), streams, log, t


def test_a_call_waits_for_the_one_before_on_another_stream(fake):
    order, s, log, t = fake
    assert order(None) == s["a"].cuda_stream and order(None) == s["a"].cuda_stream and log == []      # one stream: nothing to wait for
    order(s["b"])                       # a step on another stream than the constructor's
    order(s["b"])
    order(None)                         # new gradients on the first one, while that step may run
    order(s["c"])
    assert log == [("b", "a"), ("a", "b"), ("c", "a")] and t.used == ["b", "a", "c"]


def test_captured_calls_wait_for_nothing(fake):
    order, s, log, t = fake
    order(None)
    s["b"].capturing = True
    assert order(s["b"]) == s["b"].cuda_stream
    order(None)                         # and nothing waits for a stream that is being captured
    assert log == []
    s["b"].capturing = False
    order(s["b"])
    assert log == [("b", "a")]
    s["b"].capturing = True
    with pytest.raises(RuntimeError):
        order(None)                     # the last call's stream has become one since: an event on it would be the graph's
    s["b"].capturing = False
    order(None)
    assert log[1:] == [("a", "b")]
