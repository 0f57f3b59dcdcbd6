"""How an explainer network scales its inputs and values, without a GPU: the exact values
are stood in for."""
import warnings
from types import SimpleNamespace

import pytest
import torch

from paper_2010_13972_amd import explainer, gts


def network(monkeypatch, X, dtype=torch.float32, values=lambda rows: torch.randn(rows, 1, 4)):
    monkeypatch.setattr(gts, "shap", lambda model, rows: values(rows.shape[0]))
    m = X.shape[1]
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        return explainer.Explainer(SimpleNamespace(num_groups=1, num_features=m), X, 8, 1, dtype)


@pytest.mark.parametrize("value", [0.0, 0.3, -4e5])
def test_a_feature_without_variation_keeps_its_unit(monkeypatch, value):
    """Rows explained later may hold other values there; they stay within float16."""
    X = torch.randn(100, 3)
    X[:, 1] = value
    net = network(monkeypatch, X, torch.float16)
    later = X.clone()
    later[:, 1] += 1.0
    x = net._inputs(later)
    assert torch.isfinite(x).all()
    assert (x[:, 1] - 1.0).abs().max() <= 1e-3 and not net._inputs(X)[:, 1].any()
    want = (X - X.mean(0)) / X.std(0)
    assert torch.equal(net._inputs(X)[:, ::2], want.half()[:, ::2])


def test_one_row(monkeypatch):
    net = network(monkeypatch, torch.randn(1, 3))
    assert torch.equal(net._inputs(net.X), torch.zeros(1, 3)) and net.spread > 0


@pytest.mark.parametrize("values", [lambda rows: torch.ones(rows, 1, 2), lambda rows: torch.zeros(rows, 1, 2)])
def test_one_value(monkeypatch, values):
    """One feature and one row have no spread; neither have values that are all alike."""
    assert network(monkeypatch, torch.randn(1, 1), values=values).spread == 1.0
    assert network(monkeypatch, torch.randn(5, 1), values=values).spread == 1.0
