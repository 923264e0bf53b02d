"""Edges of the adapter calls, against the formulas in 64 bits (bounds as in the products' own tests)."""
import numpy as np
import pytest
import torch

from test_gpu_project import DEV, EPS, Case, Side, near, tokens, y_tol

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,G", [(8, 64), (24, 128), (40, 384)])
def test_a_code_stream_that_ends_with_its_last_code(windq, rows, G):
    """The padding behind the last unit is not there: trits of an odd number of bytes a row."""
    c = Case(windq, rows, 3 * G, G, 0, seed=2, only=5)
    per_unit = (G + 4) // 5 * rows
    exact = 2 * ((per_unit + 15) // 16 * 16) + per_unit
    room = torch.full((exact + 64,), 255, dtype=torch.uint8, device=DEV)        # 255 is no five trits: what is read of it would show
    room[:exact] = c.codes[:exact]
    packed = c.describe(windq, codes=room[:exact])
    for T in (1, 9, 70):
        X = tokens(T, 3 * G, torch.bfloat16, T)
        x = X.double().cpu().numpy()
        want = x @ c.w.T
        near(windq.windq_project(packed, X), want, y_tol(c, x, torch.bfloat16, want))


def three(windq, rows, cols, T, dtype, seed):
    """Three adapters beside a packed matrix: (packed, a, b, adapter_of, x, dy)."""
    g = torch.Generator().manual_seed(seed)
    c = Case(windq, rows, cols, 128, 0, dtype, seed=seed)
    a, b = (torch.randn(3, 16, cols, generator=g) / cols ** 0.5).to(dtype).to(DEV), (0.05 * torch.randn(3, rows, 16, generator=g)).to(dtype).to(DEV)
    of = torch.randint(-1, 3, (T,), generator=g).to(torch.int32).to(DEV)
    return c, a, b, of, tokens(T, cols, dtype, seed + 1), tokens(T, rows, dtype, seed + 2)


# for few tokens, for any shape, and tiles (1024 rows, 4 k-blocks: more than 512 tokens)
ROUTES = [(256, 512, 40), (256, 512, 300), (1024, 512, 700), (100, 256, 90)]


@pytest.mark.parametrize("rows,cols,T", ROUTES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_factor_that_is_not_finite_leaves_the_other_requests_alone(windq, rows, cols, T, dtype):
    c, a, b, of, x, dy = three(windq, rows, cols, T, dtype, 1)

    def both(alpha):
        ad = windq.Adapters(a, b, torch.tensor(alpha, device=DEV))
        return windq.windq_project(c.packed, x, ad, of), *windq.windq_project_grad(c.packed, dy, x, ad, of)

    clean, others = both([0.5, 2.0, 1.5]), of != 1
    for bad in (float("nan"), float("inf"), float("-inf")):
        y, dx, da, db = both([0.5, bad, 1.5])
        assert torch.equal(y[others], clean[0][others]) and torch.equal(dx[others], clean[1][others])
        assert torch.equal(da[[0, 2]], clean[2][[0, 2]]) and torch.equal(db[[0, 2]], clean[3][[0, 2]])
        assert not torch.isfinite(y[~others]).any() and not torch.isfinite(dx[~others]).any()


@pytest.mark.parametrize("T", [0, 3, 90, 700])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_an_adapter_without_tokens_has_no_gradient_whatever_its_factor(windq, T, dtype):
    c, a, b, of, x, dy = three(windq, 256, 256, T, dtype, 2)
    of[of == 1] = 0
    for bad in (float("nan"), float("inf")):
        ad = windq.Adapters(a, b, torch.tensor([0.5, bad, 1.5], device=DEV))
        _, da, db = windq.windq_project_grad(c.packed, dy, x, ad, of)
        assert torch.all(da[1] == 0) and torch.all(db[1] == 0) and torch.all(torch.isfinite(da)) and torch.all(torch.isfinite(db))


@pytest.mark.parametrize("rows,cols,T", ROUTES)
@pytest.mark.parametrize("top", [3.4e38, -3.4e38])
def test_the_largest_fp32_values_are_values(windq, rows, cols, T, top):
    """fp32 above bfloat16's largest value is finite: in an adapter (the other requests keep their bits, its own follow the formula) and in h."""
    c, a, b, of, x, dy = three(windq, rows, cols, T, torch.float32, 3)

    def y_of(a, b):
        return windq.windq_project(c.packed, x, windq.Adapters(a, b), of)

    clean, others = y_of(a, b), of != 1
    a2, b2 = a.clone(), b.clone()
    a2[1, 2] *= 1e-30
    b2[1, 7, 2] = top
    b2[1, rows - 1, 2] = top / 1.0000001
    y = y_of(a2, b2)
    assert torch.equal(y[others], clean[others])
    x64, mine = x.double().cpu().numpy(), (~others).cpu().numpy()
    A, B = a2[1].double().cpu().numpy(), b2[1].double().cpu().numpy()
    want, mag = x64[mine] @ c.w.T + x64[mine] @ A.T @ B.T, np.abs(x64[mine]) @ c.mag.T + np.abs(x64[mine]) @ np.abs(A).T @ np.abs(B).T
    near(y[~others], want, EPS * mag)
    # the same for h: an A whose sums come close to the largest value, a B that brings them back
    a3, b3 = torch.zeros_like(a), b.clone()
    a3[:, :, 0] = top
    x1 = x.clone()
    x1[:, 0] = 1.0
    b3 *= 1e-20
    y = windq.windq_project(c.packed, x1, windq.Adapters(a3, b3), of)
    x64, on = x1.double().cpu().numpy(), (of >= 0).cpu().numpy()
    B = b3.double().cpu().numpy()[np.maximum(of.cpu().numpy(), 0)]
    h = float(np.float32(top)) * np.ones(16)
    side = (B @ h) * on[:, None]
    near(y, x64 @ c.w.T + side, EPS * (np.abs(x64) @ c.mag.T + np.abs(B) @ np.abs(h) * on[:, None]))
