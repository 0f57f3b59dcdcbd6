"""The large products in float16: its kernels are compiled apart from bfloat16's, with the
same plan."""
import pytest
import torch

import test_gpu_nn_linear as products
from paper_2010_13972_amd import nn

pytestmark = pytest.mark.gpu


def test_shapes_take_every_tile():
    """Each product in each of float16's tiles of 128 rows and more, and each tile with split
    sums and without."""
    seen = {(p, c["tile_m"], c["tile_n"], c["splits"] > 1) for p, shapes in products.LARGE.items()
            for s in shapes for c in [nn.linear_config(*s, torch.float16, p)]}
    for tile in ((128, 128), (192, 256), (256, 256)):
        assert {s[0] for s in seen if s[1:3] == tile} == set(products.LARGE), tile
        assert {s[3] for s in seen if s[1:3] == tile} == {False, True}, tile


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("product,shape", [(p, s) for p in products.LARGE for s in products.LARGE[p]],
                         ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v)))
def test_large(product, shape, pad):
    products.test_large(product, shape, pad, torch.float16)


@pytest.mark.parametrize("shape", [(10000, 1024, 4096), (4096, 512, 2048), (4096, 2048, 512)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_gradients_of_a_training_batch(shape, dtype):
    """All three gradients with an activation, against 64 bits on the device."""
    rows, k, n = shape
    print("training batch", shape, dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    dy, x, w, pre = ((torch.randn(r, c, generator=g, device="cuda") * std).to(dtype)
                     for r, c, std in ((rows, n, 1.0), (rows, k, 1.0), (n, k, k ** -0.5), (rows, n, 1.0)))
    got = nn.linear_backward(dy, x, w, pre=pre, act="gelu")
    at = [t.double() for t in (dy, x, w, pre)]
    want = products.backward_want(*at, "gelu")
    for value, v, t, name in zip(got, want[1:], products.backward_tols(dtype, *at, "gelu", want), ("dx", "dw", "db")):
        products.ref.assert_within(value, v, t, f"{shape} {dtype} {name}")
