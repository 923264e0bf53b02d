"""The adapter products where offsets pass 32 bits: tokens x columns, and windows of tensors with long rows.  Against the formulas in 64 bits for tokens on both
sides of the limits, and bit for bit against the same values lying close together."""
import numpy as np
import pytest
import torch

from test_gpu_project import DEV, EPS, Case, Side, near, tokens, y_tol

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def memory():
    """What a test took goes back, for the tests behind it."""
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,masked", [(BF, False), (F32, False), (BF, True), (F32, True)])
def test_more_than_two_to_the_31_activations(windq, dtype, masked):
    rows, cols, T = 256, 65536, 33001                    # 2^31 values end inside token 32768
    c = Case(windq, rows, cols, 128, 64, masked=masked, seed=1)
    g = torch.Generator(device=DEV).manual_seed(1)
    X = torch.empty(T, cols, dtype=dtype, device=DEV)
    for part in X.split(4096):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV))
    some = [0, 1, 5000, 16383, 16384, 16385, 32766, 32767, 32768, 32769, T - 2, T - 1]
    a, b = (torch.randn(2, 8, cols, generator=g, device=DEV) / 256).to(dtype), (0.05 * torch.randn(2, rows, 8, generator=g, device=DEV)).to(dtype)
    of = torch.randint(0, 2, (T,), generator=g, device=DEV, dtype=torch.int32)
    h = torch.empty(T, 8, device=DEV)
    y = windq.windq_project(c.packed, X, windq.Adapters(a, b), of, h=h)
    x, k = X[some].double().cpu().numpy(), of[some].long().cpu().numpy()
    A, B = a.double().cpu().numpy()[k], b.double().cpu().numpy()[k]
    hw, hm = np.matmul(A, x[:, :, None])[:, :, 0], np.matmul(np.abs(A), np.abs(x)[:, :, None])[:, :, 0]
    near(h[some], hw, EPS * hm)
    want, ym = x @ c.w.T + np.matmul(B, hw[:, :, None])[:, :, 0], np.matmul(np.abs(B), hm[:, :, None])[:, :, 0]
    near(y[some], want, y_tol(c, x, dtype, want, ym))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,masked", [(7, False), (60, False), (700, False), (700, True)])
def test_windows_of_long_rows(windq, dtype, T, masked):
    """X, dY, Y, dX and W as windows of tensors with rows of millions of values: the bits of the same values in close rows."""
    rows, cols = 1024, 512
    wide = {7: 1 << 30, 60: 1 << 26, 700: 1 << 23}[T]    # the last tokens' offsets pass 2^31, or 2^32
    c = Case(windq, rows, cols, 128, 0, dtype, masked=masked, seed=2)
    s = Side(windq, 3, 16, rows, cols, dtype, T, seed=3)
    X, dY = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    y = windq.windq_project(c.packed, X, s.adapters, s.of_dev)
    grads = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev)

    def window(t):
        w = torch.empty(t.shape[0], wide, dtype=t.dtype, device=DEV)[:, wide - 2048:][:, 8:8 + t.shape[1]]
        return w.copy_(t)

    xw = window(X)
    out = window(torch.zeros_like(y))
    windq.windq_project(c.packed, xw, s.adapters, s.of_dev, out=out)
    assert torch.equal(out, y)
    del out
    dyw, dxw = window(dY), window(torch.zeros_like(X))
    got = windq.windq_project_grad(c.packed, dyw, xw, s.adapters, s.of_dev, outs=(dxw, None, None))
    assert all(torch.equal(p, q) for p, q in zip(got, grads))
    del xw, dyw, dxw, got
    if T == 700:
        W = torch.empty(rows, 1 << 22, dtype=dtype, device=DEV)[:, (1 << 22) - 1024:][:, :cols]
        packed = c.describe(windq, W=W.copy_(c.W))
        assert torch.equal(windq.windq_project(packed, X, s.adapters, s.of_dev), y)
        assert torch.equal(windq.windq_project_grad(packed, dY, X, s.adapters, s.of_dev)[0], grads[0])
