"""gts_grad_clip on gradients whose squares leave the range of 32 bits while their norm does
not.  Squares of 32-bit values are exact in 64 bits, so the norm is off by its rounding and
by some 2^-50; the factor by that and three roundings more."""
import math

import pytest
import torch

from nn_reference import U32, d
from paper_2010_13972_amd import nn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [2e19, 1e36, 3e-23, 1e-30, 1e-38])
@pytest.mark.parametrize("counts", [(3,), (9000, 1), (20000, 70, 300)], ids=lambda c: "+".join(map(str, c)))
def test_norm_of_large_and_tiny_gradients(dtype, size, counts):
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    g = torch.Generator().manual_seed(1)
    grads = [((torch.rand(n, generator=g) + 0.5) * size).to(dtype).cuda() for n in counts]
    norm = math.sqrt(sum(float((d(t) ** 2).sum()) for t in grads))
    clip = nn.grad_clip(grads, 2.0)
    factor = min(1.0, 2.0 / (norm + 1e-6))
    assert abs(float(clip[0]) - norm) <= 2 * U32 * norm + 2.0 ** -149
    assert abs(float(clip[1]) - factor) <= 6 * U32 * factor
    # the step they clip is a step: no value is lost, none is NaN
    p = [torch.zeros(n, device="cuda") for n in counts]
    s = nn.adamw_state(p)
    nn.adamw_step(p, grads, s.m, s.v, step=1, lr=1.0, eps=1e-8, clip=clip)
    assert all(torch.isfinite(t).all() for t in p)
    for t, q in zip(grads, p):
        want = d(t) * float(clip[1])
        want = -want / (want.abs() + 1e-8)
        small = d(t).abs() * float(clip[1]) < 1e-18   # whose squares AdamW's 32-bit moments do not hold
        assert ((d(q) - want).abs() <= 1e-5 * want.abs() + small * 1e-9).all()


def test_a_norm_past_32_bits():
    clip = nn.grad_clip([torch.full((4,), 3e38, device="cuda")], 1.0)
    assert float(clip[0]) == math.inf and math.isnan(float(clip[1]))
