"""A served explainer network whose network object is gone."""
import gc
import weakref

import pytest
import torch

from paper_2010_13972_amd import explainer, gts, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_serves_without_its_network(dtype):
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    model = gts.prepare(synth.workload("tiny").ensemble, "f32")
    X = torch.from_numpy(synth.sweep_rows("tiny", 512)).cuda()
    net = explainer.Explainer(model, X, width=64, blocks=2, dtype=dtype)
    want = [net.explain(X[i * 30:(i + 1) * 30]) for i in range(4)]
    read = [weakref.ref(t) for t in (*net.weights.values(), net.mean, net.dev, net.bias)]
    serve = net.server(30)
    del net
    gc.collect()
    assert all(r() is not None for r in read)
    # what was freed has been taken by others
    other = [torch.full((64, 64), float("nan"), device="cuda", dtype=dtype) for _ in range(200)]
    for i in range(4):
        assert torch.equal(serve(X[i * 30:(i + 1) * 30]), want[i]), i
    del serve, other
    gc.collect()
    assert all(r() is None for r in read)
