"""Where calls with ``stream=`` take their memory from, on a stand-in for torch: no GPU."""

import contextlib

import pytest


class Memory:
    def __init__(self, pool):
        self.pool, self.noted = pool, []

    def record_stream(self, stream):
        self.noted.append(stream)


class Torch:
    """torch.empty and the stream functions that it answers to."""

    def __init__(self):
        self.stack = ["the current stream"]
        self.cuda = self
        self.taken = []

    def empty(self, shape, dtype=None, device=None):
        self.taken.append(Memory(self.stack[-1]))
        return self.taken[-1]

    @contextlib.contextmanager
    def stream(self, stream):
        self.stack.append(stream)
        yield
        self.stack.pop()

    def current_stream(self, device=None):
        return self.stack[-1]


@pytest.fixture
def kd(monkeypatch):
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    fake = Torch()
    monkeypatch.setattr(kashin, "_torch", lambda: fake)
    return kashin


def test_an_output_comes_from_the_pool_of_the_stream_that_writes_it(kd):
    t = kd._new("side", (2, 3), None, "cuda")
    assert t.pool == "side" and t.noted == ["the current stream"]
    t = kd._new(None, (2, 3), None, "cuda")
    assert t.pool == "the current stream" and not t.noted
    t = kd._new("the current stream", (2, 3), None, "cuda")
    assert t.pool == "the current stream" and not t.noted
