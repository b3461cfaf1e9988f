"""examples/serve_batch.py without a GPU: what its server keeps, counts and refuses, with the step and the graph capture stood in for."""
import contextlib
import gc
import os
import sys
import weakref

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from serve_batch import Server  # noqa: E402


class Graph:
    """Runs nothing when replayed."""

    def replay(self):
        pass


@pytest.fixture
def host(monkeypatch):
    """A server of three sequences whose buffers are host tensors and whose step only notes its arguments; captures do nothing."""
    class Stream:
        def wait_stream(self, other):
            pass
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "CUDAGraph", Graph)

    class Host(Server):
        def __init__(self):
            self.lens, self.table, self.longest = torch.zeros(3, dtype=torch.int32), torch.arange(3, dtype=torch.int32).view(3, 1), 9000
            self.cached, self.given, self.calls = [0, 0, 0], [], []

        def buffers(self, tokens):
            return {n: torch.zeros(tokens, 4) for n in ("qkv", "q", "o", "y", "x", "h", "scores", "ws")}

        def step(self, b, embedded, pos, seq, rows, lens, max_len):
            self.given += [weakref.ref(t) for t in (*b.values(), lens, embedded)]
            self.calls.append((embedded.clone(), pos.clone(), None if seq is None else seq.clone(), rows.clone(), lens.clone(), max_len))
            b["x"].copy_(embedded)
            return b["x"]
    server = Host()

    @contextlib.contextmanager
    def graph(g):                                    # what is captured is not run
        before = server.lens.clone()
        yield
        server.lens.copy_(before)
    monkeypatch.setattr(torch.cuda, "graph", graph)
    return server


@pytest.mark.parametrize("eager", [True, False])
def test_a_decoder_keeps_what_its_graph_reads_and_writes(host, eager):
    token = host.decoder(torch.zeros(3, 4), eager)
    token()
    given, server = host.given, weakref.ref(host)
    del host.given
    gc.collect()
    assert given and all(r() is not None for r in given)
    del token
    gc.collect()
    assert all(r() is None for r in given) and server() is host      # and no longer than it lives itself


def test_prompts_go_in_parts(host):
    host.prompt(torch.zeros(9, 4), [4, 0, 5])
    host.calls.clear()
    embedded = torch.randn(4097 + 4096, 4)
    x = host.prompt(embedded, [5000, 3, 3190])
    assert torch.equal(x, embedded) and host.lens.tolist() == host.cached == [5004, 3, 3195]
    assert [len(c[0]) for c in host.calls] == [4096, 4096, 1]
    pos, seq, rows, lens = (torch.cat([c[i] for c in host.calls]) for i in (1, 2, 3, 4))
    assert pos.tolist() == [*range(4, 5004), *range(3), *range(5, 3195)] and torch.equal(lens, pos + 1)
    assert seq.tolist() == [0] * 5000 + [1] * 3 + [2] * 3190 and torch.equal(rows[:, 0], seq)
    assert len(host.prompt(torch.zeros(0, 4), [0, 0, 0])) == 0 and len(host.calls) == 3


def test_what_there_is_no_room_for_is_refused(host):
    host.prompt(torch.zeros(9000, 4), [8999, 0, 1])
    state, calls = (host.lens.tolist(), list(host.cached)), len(host.calls)
    for tokens, counts in ((2, [2, 0, 0]), (3, [1, 1]), (1, [1]), (4, [1, 1, 1]), (0, [1, -1, 0]), (9001, [0, 9001, 0])):
        with pytest.raises(ValueError):
            host.prompt(torch.zeros(tokens, 4), counts)
    assert (host.lens.tolist(), host.cached) == state and len(host.calls) == calls
    token = host.decoder(torch.zeros(3, 4), eager=True)
    token()
    assert host.lens.tolist() == host.cached == [9000, 1, 2]
    for t in (token, host.decoder(torch.zeros(3, 4))):
        with pytest.raises(ValueError, match="no room"):
            t()
    assert host.lens.tolist() == host.cached == [9000, 1, 2]


def test_a_step_that_fails_moves_no_length(host):
    def fails(*args):
        raise RuntimeError("step")
    token = host.decoder(torch.zeros(3, 4), eager=True)
    token()
    host.step = fails
    for run in (token, lambda: host.prompt(torch.zeros(2, 4), [1, 0, 1])):
        with pytest.raises(RuntimeError, match="step"):
            run()
        assert host.lens.tolist() == host.cached == [1, 1, 1]
