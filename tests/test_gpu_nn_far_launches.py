"""Products of more workgroups than a launch has along one axis (2^32 work-items): very many
rows of few columns, very many outputs.  Values are small whole numbers whose sums are
exact, so that the results are equal to torch's."""
import pytest
import torch

from paper_2010_13972_amd import nn

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def device():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    yield
    torch.cuda.empty_cache()


def whole(shape, seed, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


def ends(n, at=1000):
    """Where an axis begins, where its launch would end and where it ends itself."""
    limit = 64 * ((1 << 32) // 512)
    return [slice(0, at), slice(min(limit, n) - at, min(limit + at, n)), slice(n - at, n)]


@pytest.mark.parametrize("inputs,outputs,dtype", [(1, 1, BF16), (8, 3, BF16), (1, 2, torch.float32)])
def test_many_rows(inputs, outputs, dtype):
    rows = 560_000_003
    print("many rows", inputs, outputs, dtype, flush=True)
    x, w = whole((rows, inputs), 1, dtype), whole((outputs, inputs), 2, dtype)
    b = whole((outputs,), 3, dtype)
    y = nn.linear(x, w, b)
    for i in range(0, rows, 1 << 26):
        part = x[i:i + (1 << 26)]
        want = b + sum(part[:, k:k + 1] * w[:, k] for k in range(inputs))
        assert torch.equal(y[i:i + (1 << 26)], want), i
    del y
    dy = torch.zeros(rows, outputs, dtype=dtype, device="cuda")
    for n, at in enumerate(ends(rows, 20)):
        dy[at] = whole((dy[at].shape[0], outputs), 4 + n, dtype)
    dx, dw, db = nn.linear_backward(dy, x, w)
    for at in ends(rows):
        assert torch.equal(dx[at].float(), dy[at].float() @ w.float()), at
    some = torch.cat([torch.arange(rows, device="cuda")[at] for at in ends(rows, 20)])
    assert torch.equal(dw.float(), dy[some].float().T.contiguous() @ x[some].float())
    assert torch.equal(db.float(), dy[some].float().sum(0))


def test_many_outputs():
    outputs, inputs = 150_000_001, 8
    print("many outputs", flush=True)
    x, w, b = whole((2, inputs), 1), whole((outputs, inputs), 2), whole((outputs,), 3)
    y = nn.linear(x, w, b)
    for i in range(0, outputs, 1 << 25):
        at = slice(i, i + (1 << 25))
        want = sum(x[:, k:k + 1] * w[at, k] for k in range(inputs)) + b[at]
        assert torch.equal(y[:, at], want), i
    dy = torch.zeros(2, outputs, dtype=BF16, device="cuda")
    cols = [slice(0, 20), slice((1 << 27) - 10, (1 << 27) + 10), slice(outputs - 20, outputs)]
    for n, at in enumerate(cols):
        dy[:, at] = whole((2, 20), 4 + n)
    dx, dw, db = nn.linear_backward(dy, x, w)
    want = sum(dy[:, at].float() @ w[at].float() for at in cols)
    assert torch.equal(dx.float(), want)
    for at in cols + [slice(5000, 6000)]:
        assert torch.equal(dw[at].float(), dy[:, at].float().T.contiguous() @ x.float())
        assert torch.equal(db[at].float(), dy[:, at].float().sum(0))
    assert not dw[20:(1 << 27) - 10].any() and not db[(1 << 27) + 10:-20].any()
