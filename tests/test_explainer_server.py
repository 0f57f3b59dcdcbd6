"""What a served explainer network keeps alive, without a GPU: the graph is stood in for."""
import contextlib
import gc
import weakref

import torch

from paper_2010_13972_amd import explainer


class _Stream:
    def wait_stream(self, other):
        pass


class _Graph:
    replays = 0

    def replay(self):
        self.replays += 1


def test_a_server_keeps_what_its_graph_reads(monkeypatch):
    """A graph holds addresses: the weights, the inputs' scaling and the bias have to outlive
    the network object while the function that replays the graph is there."""
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", _Stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "CUDAGraph", _Graph)
    monkeypatch.setattr(torch.cuda, "graph", lambda g: contextlib.nullcontext())
    monkeypatch.setattr(explainer.Explainer, "explain", lambda self, X: torch.zeros(X.shape[0], 1, 4))
    net = explainer.Explainer.__new__(explainer.Explainer)
    net.X, net.shape = torch.zeros(5, 3), (1, 3)
    net.weights = {"w_in": torch.ones(4, 3), "w_out": torch.ones(3, 4)}
    net.mean, net.dev, net.bias = torch.zeros(3), torch.ones(3), torch.zeros(1)
    read = [weakref.ref(t) for t in (*net.weights.values(), net.mean, net.dev, net.bias)]
    serve = net.server(2)
    del net
    gc.collect()
    assert all(r() is not None for r in read)
    assert serve(torch.zeros(2, 3)).shape == (2, 1, 4)
    del serve
    gc.collect()
    assert all(r() is None for r in read)
