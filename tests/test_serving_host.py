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
    monkeypatch.setattr(torch.cuda, "graph", lambda g: contextlib.nullcontext())

    class Host(Server):
        def __init__(self):
            self.lens, self.table, self.longest = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32), 60
            self.given = []                          # weak references to what each decoder's captures were given

        def buffers(self, tokens):
            return {n: torch.zeros(tokens, 4) for n in ("qkv", "q", "o", "y", "x", "h", "scores", "ws")}

        def step(self, b, embedded, pos, seq, rows, lens, max_len):
            self.given += [weakref.ref(t) for t in (*b.values(), pos, embedded)]
            return b["x"]
    return Host()


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
