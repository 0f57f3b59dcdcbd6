"""Training of the explainer network in float16: the gradients of a batch as the command
takes it, and overflows."""
import pytest
import torch

from paper_2010_13972_amd import explainer, gts, nn, synth

pytestmark = pytest.mark.gpu


def networks(name, rows, *dtypes):
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    model = gts.prepare(synth.workload(name).ensemble, "f32")
    X = torch.from_numpy(synth.sweep_rows(name, rows)).cuda()
    return X, [explainer.Explainer(model, X, width=512, blocks=2, dtype=t) for t in dtypes]


def assert_same_moments(got, want, tol):
    """The first moments of two networks, tensor by tensor, in their 2-norms."""
    for name, a, t in zip(want.names, nn.state_offsets(want.master)[0], want.master):
        p, q = (n.state.m[a:a + t.numel()].double() for n in (want, got))
        assert (q - p).norm() <= tol * p.norm(), (name, float((q - p).norm() / p.norm()))


@pytest.mark.parametrize("name", ["tiny", "covtype_med", "wide"])
def test_gradients_of_a_batch(name):
    """The first step's moments, a tenth of the clipped gradients, against float32's.  From
    rows to the input layer's gradient some 35 values are rounded one after the other, each
    by up to 2^-11 of itself: 0.018 where all go one way."""
    X, (f32, f16) = networks(name, 4096, torch.float32, torch.float16)
    for net in (f32, f16):
        net.train_step(X, 1e-3)
    assert_same_moments(f16, f32, 0.018)


def test_overflow():
    """Gradients past 65504 change no weight and no moment but lower the scale; the next
    step's moments are those of any scale."""
    X, (f32, f16) = networks("tiny", 1024, torch.float32, torch.float16)
    before = [t.clone() for t in f16.master]
    f16.loss_scale.fill_(2.0 ** 18)
    f16.train_step(X, 0.0)
    assert not f16.state.m.any() and not f16.state.v.any()
    assert all(torch.equal(a, b) for a, b in zip(f16.master, before))
    scale = float(f16.loss_scale)
    assert 0 < scale <= explainer._SCALE
    for net in (f32, f16):
        net.train_step(X, 0.0)
    # both took one step; the float16 network's is its second by number, moments know no number
    assert_same_moments(f16, f32, 0.018)
    f16.loss_scale.fill_(scale / 4)
    f16.state.m.zero_()
    f16.train_step(X, 0.0)
    assert_same_moments(f16, f32, 0.018)
    assert scale / 4 < float(f16.loss_scale) < scale / 2
