"""Edges of the adapter calls, against the formulas in 64 bits (bounds as in the products' own tests)."""
import numpy as np
import pytest
import torch

from test_gpu_project import DEV, EPS, Case, Side, near, tokens, y_tol

pytestmark = pytest.mark.gpu


@pytest.fixture
def much_memory():
    """What the test took goes back, for the tests behind it."""
    yield
    torch.cuda.empty_cache()


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


def test_more_tokens_times_ranks_than_one_launch_takes(windq):
    """fp32, 2^26 and some: h of the first and last tokens, and of those on both sides of a launch's end."""
    rows, cols, T, r = 8, 64, (1 << 19) + 77, 128
    c = Case(windq, rows, cols, 64, 0, torch.float32, seed=3)
    g = torch.Generator(device=DEV).manual_seed(1)
    X, dY = torch.randn(T, cols, generator=g, device=DEV), torch.randn(T, rows, generator=g, device=DEV)
    a, b = torch.randn(2, r, cols, generator=g, device=DEV) / 8, 0.05 * torch.randn(2, rows, r, generator=g, device=DEV)
    of = torch.randint(0, 2, (T,), generator=g, device=DEV, dtype=torch.int32)
    h = torch.full((T, r), float("nan"), device=DEV)
    ad = windq.Adapters(a, b)
    y = windq.windq_project(c.packed, X, ad, of, h=h)
    dx = windq.windq_project_grad(c.packed, dY, X, ad, of, h=h)[0]
    end = ((1 << 24) - 1) // 32                          # tokens of a launch
    some = [*range(40), *range(end - 40, end + 40), *range(T - 90, T)]
    x, dy, k = X[some].double().cpu().numpy(), dY[some].double().cpu().numpy(), of[some].long().cpu().numpy()
    A, B = a.double().cpu().numpy()[k], b.double().cpu().numpy()[k]
    hw, hm = np.matmul(A, x[:, :, None])[:, :, 0], np.matmul(np.abs(A), np.abs(x)[:, :, None])[:, :, 0]
    near(h[some], hw, EPS * hm)
    near(y[some], x @ c.w.T + np.matmul(B, hw[:, :, None])[:, :, 0], EPS * (np.abs(x) @ c.mag.T + np.matmul(np.abs(B), hm[:, :, None])[:, :, 0]))
    d, dm = np.matmul(dy[:, None, :], B), np.matmul(np.abs(dy)[:, None, :], np.abs(B))
    near(dx[some], dy @ c.w + np.matmul(d, A)[:, 0], EPS * (np.abs(dy) @ c.mag + np.matmul(dm, np.abs(A))[:, 0]))


def test_more_adapters_than_one_launch_takes(windq, much_memory):
    """2^20 adapters, three of them in use: the first, one in the middle and the last; every other one's gradient is zero."""
    n, r, rows, cols, T = 1 << 20, 8, 64, 1024, 100
    c = Case(windq, rows, cols, 128, 0, seed=3)
    g = torch.Generator().manual_seed(2)
    a, b = torch.zeros(n, r, cols, dtype=torch.bfloat16, device=DEV), torch.zeros(n, rows, r, dtype=torch.bfloat16, device=DEV)
    used = [0, n // 2 + 5, n - 1]
    for k in used:
        a[k], b[k] = (torch.randn(r, cols, generator=g) / 32).to(DEV), (0.05 * torch.randn(rows, r, generator=g)).to(DEV)
    of = torch.tensor(used)[torch.randint(0, 3, (T,), generator=g)].to(torch.int32)
    X, dY = tokens(T, cols, torch.bfloat16, 3), tokens(T, rows, torch.bfloat16, 4)
    ad = windq.Adapters(a, b)
    y = windq.windq_project(c.packed, X, ad, of.to(DEV))
    da, db = (torch.full(t.shape, float("nan"), device=DEV) for t in (a, b))
    windq.windq_project_grad(c.packed, dY, X, ad, of.to(DEV), outs=(None, da, db))
    x, dy = X.double().cpu().numpy(), dY.double().cpu().numpy()
    want, tol = x @ c.w.T, np.abs(x) @ c.mag.T
    for k in used:
        at = np.flatnonzero(of.numpy() == k)
        A, B = a[k].double().cpu().numpy(), b[k].double().cpu().numpy()
        h, hm = x[at] @ A.T, np.abs(x[at]) @ np.abs(A).T
        want[at] += h @ B.T
        tol[at] += hm @ np.abs(B).T
        near(da[k], (dy[at] @ B).T @ x[at], EPS * ((np.abs(dy[at]) @ np.abs(B)).T @ np.abs(x[at])))
        near(db[k], dy[at].T @ h, EPS * (np.abs(dy[at]).T @ hm))
    near(y, want, EPS * tol + 2.0 ** -8 * 1.001 * np.abs(want) + 2.0 ** -16 * tol)
    for t in (da, db):
        t[used] = 0
        for part in t.split(1 << 16):
            assert not part.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_plan_of_skip_units_alone(windq, dtype):
    """No codes at all, and none given."""
    c = Case(windq, 96, 256, 64, 0, seed=2, only=0)
    packed = c.describe(windq, codes=torch.empty(0, dtype=torch.uint8, device=DEV))
    for T in (1, 40, 200):
        X, dY = tokens(T, 256, dtype, T), tokens(T, 96, dtype, T + 1)
        x, dy = X.double().cpu().numpy(), dY.double().cpu().numpy()
        near(windq.windq_project(packed, X), x @ c.w.T, y_tol(c, x, dtype, x @ c.w.T))
        near(windq.windq_project_grad(packed, dY)[0], dy @ c.w, EPS * (np.abs(dy) @ c.mag) + (2.0 ** -8 * 1.001 * np.abs(dy @ c.w) if dtype == torch.bfloat16 else 0.0))


def test_the_example_with_fewer_tokens_than_it_serves(windq):
    from paper_2605_26660_amd import adapt

    first, last, differs = adapt.run(rows=64, cols=128, chunk_w=64, steps=2, tokens=16, rank=8)
    assert len(first) == len(last) == 3 and differs < 3 * 2.0 ** -8
