"""What one token, one row, one request may not change of the others', on every route (kernels by the rules that test_gpu_project_routes checks)."""
import numpy as np
import pytest
import torch

from test_gpu_project import DEV, Case, Side, tokens

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# tokens, rows, cols, chunk width, unit rows, mask: few tokens as they lie and laid out, one and two fragments; any shape; tiles; the way back split and whole
SHAPES = [(7, 256, 512, 128, 0, False), (30, 256, 512, 128, 0, False), (200, 256, 512, 128, 0, False), (300, 200, 320, 32, 0, False), (300, 256, 512, 128, 0, True),
          (700, 1024, 512, 128, 0, False), (700, 1024, 768, 256, 128, False), (2000, 136, 4096, 128, 0, False)]


@pytest.mark.parametrize("T,rows,cols,G,unit_rows,masked", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_other_requests_values_change_nothing(windq, T, rows, cols, G, unit_rows, masked, dtype):
    """X, dY and the adapters of some requests change (finite values, the same grouping): the others' results keep their bits."""
    c = Case(windq, rows, cols, G, unit_rows, masked=masked, seed=1)
    s = Side(windq, 5, 24, rows, cols, dtype, T, seed=3, plain=True)
    X, dY = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    a, b = s.a.to(DEV), s.b.to(DEV)

    def both(X, dY, a, b):
        ad = windq.Adapters(a, b)
        return windq.windq_project(c.packed, X, ad, s.of_dev), *windq.windq_project_grad(c.packed, dY, X, ad, s.of_dev)

    first = both(X, dY, a, b)
    theirs = (s.of_dev == 1) | (s.of_dev == 3)
    X2, dY2, a2, b2 = X.clone(), dY.clone(), a.clone(), b.clone()
    X2[theirs] = tokens(T, cols, dtype, 11, 30.0)[theirs]
    dY2[theirs] = tokens(T, rows, dtype, 12, 30.0)[theirs]
    a2[[1, 3]], b2[[1, 3]] = -3 * a[[1, 3]], 5 * b[[3, 1]]
    then = both(X2, dY2, a2, b2)
    assert all(torch.equal(x[~theirs], y[~theirs]) for x, y in zip(first[:2], then[:2]))
    assert all(torch.equal(x[[0, 2, 4]], y[[0, 2, 4]]) for x, y in zip(first[2:], then[2:]))
    if theirs.any():
        assert not torch.equal(first[0][theirs], then[0][theirs]) and not torch.equal(first[1][theirs], then[1][theirs])


@pytest.mark.parametrize("T,rows,cols,G,unit_rows,masked", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_is_not_finite_reaches_its_own_results_alone(windq, T, rows, cols, G, unit_rows, masked, dtype):
    """Infinities and NaN in X, in a scale, an offset and a skip weight: their tokens' and rows' results as the formula has them, the others' bits kept."""
    c = Case(windq, rows, cols, G, unit_rows, masked=masked, seed=1)
    X = tokens(T, cols, dtype, 3)
    clean = windq.windq_project(c.packed, X)
    x2 = X.clone()
    x2[1, cols // 3], x2[2, cols - 1], x2[4, 5] = float("inf"), float("-inf"), float("nan")
    W, scale, offset = c.W.clone(), c.scale.clone(), c.offset.clone()
    nc, act = cols // G, c.action.tolist()
    unit = [next((j for j in range(nc) if act[j] == a), None) for a in (1, 2, 5, 0)]      # of the first row block, a treatment each
    bad_rows = {}
    for row, (u, which) in enumerate(zip(unit, ("scale", "offset", "scale", "W"))):
        if u is None:
            continue
        value = (float("inf"), float("nan"), float("nan"), float("inf"))[row]
        if which == "W":
            W[row, u * G + 3] = value
        else:
            (scale if which == "scale" else offset).view(-1)[u * c.R_u + row] = value
        bad_rows[row] = (u, which, value)
    got = windq.windq_project(c.describe(windq, W=W, scale=scale, offset=offset), x2)
    fine_t = [t for t in range(T) if t not in (1, 2, 4)]
    fine_r = [r for r in range(rows) if r not in bad_rows]
    assert torch.equal(got[fine_t][:, fine_r], clean[fine_t][:, fine_r])
    g = got.double().cpu().numpy()
    with np.errstate(all="ignore"):
        for t, col in ((1, cols // 3), (2, cols - 1)):
            want = c.w[fine_r, col] * float(x2[t, col])      # a weight that is 0 (protected ones are left out: w = 0 there, and no product)
            if masked:
                continue
            assert np.array_equal(np.isnan(want), np.isnan(g[t, fine_r])) and np.array_equal(want[~np.isnan(want)], g[t, fine_r][~np.isnan(want)])
    assert np.all(np.isnan(g[4][fine_r])) or masked
    for row, (u, which, value) in bad_rows.items():
        if masked:
            continue
        if which == "W":                                    # an infinite weight: infinite with the sign of its x
            want = value * X[fine_t, u * G + 3].double().cpu().numpy()
            assert np.array_equal(g[fine_t, row], want)
        else:                                               # a scale or offset that is not finite: nothing finite is left of a sum with it
            assert not np.isfinite(g[fine_t, row]).any()


@pytest.mark.parametrize("T,rows,cols,G,unit_rows,masked", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_windows_of_wider_tensors(windq, T, rows, cols, G, unit_rows, masked, dtype):
    """Column windows give the same bits, and nothing beside them is written."""
    c = Case(windq, rows, cols, G, unit_rows, masked=masked, seed=5)
    s = Side(windq, 4, 16, rows, cols, dtype, T, seed=2)
    X, dY = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    y = windq.windq_project(c.packed, X, s.adapters, s.of_dev)
    grads = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev)
    wide_x, wide_dy = (torch.full((T, n + 24), float("nan"), device=DEV, dtype=dtype) for n in (cols, rows))
    wide_x[:, 8:8 + cols], wide_dy[:, 3:3 + rows] = X, dY
    out, dx = (torch.full((T, n + 7), 7.0, device=DEV, dtype=dtype) for n in (rows, cols))
    windq.windq_project(c.packed, wide_x[:, 8:8 + cols], s.adapters, s.of_dev, out=out[:, 5:5 + rows])
    got = windq.windq_project_grad(c.packed, wide_dy[:, 3:3 + rows], wide_x[:, 8:8 + cols], s.adapters, s.of_dev, outs=(dx[:, 1:1 + cols], None, None))
    assert torch.equal(out[:, 5:5 + rows], y) and all(torch.equal(p, q) for p, q in zip(got, grads))
    assert torch.all(out[:, :5] == 7) and torch.all(out[:, 5 + rows:] == 7) and torch.all(dx[:, :1] == 7) and torch.all(dx[:, 1 + cols:] == 7)


@pytest.mark.parametrize("T,rows,cols,G,unit_rows,masked", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradients_that_are_not_finite_stay_with_their_token_and_adapter(windq, T, rows, cols, G, unit_rows, masked, dtype):
    """dY and X of two tokens are not finite, one with an adapter and one without: the other tokens' dX and the other adapters' gradients keep their bits."""
    c = Case(windq, rows, cols, G, unit_rows, masked=masked, seed=1)
    s = Side(windq, 4, 16, rows, cols, dtype, T, seed=2, plain=True)
    of = s.of_dev.clone()
    of[1], of[3], of[5] = 2, -1, 0
    X, dY = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    first = windq.windq_project_grad(c.packed, dY, X, s.adapters, of)
    for bad in (float("nan"), float("inf")):
        X2, dY2 = X.clone(), dY.clone()
        dY2[1, rows // 2], X2[1, 7], dY2[3, 0], X2[3, cols - 1] = bad, bad, bad, bad
        then = windq.windq_project_grad(c.packed, dY2, X2, s.adapters, of)
        others = [t for t in range(T) if t not in (1, 3)]
        assert torch.equal(first[0][others], then[0][others])
        assert all(torch.equal(x[[0, 1, 3]], y[[0, 1, 3]]) for x, y in zip(first[1:], then[1:]))
        assert not torch.isfinite(then[1][2]).all() and not torch.isfinite(then[2][2]).all() and not torch.isfinite(then[0][[1, 3]]).all(1).any()


@pytest.mark.parametrize("T,rows,cols,G,unit_rows,masked", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_graph_of_both_ways_replays_what_eager_calls_give(windq, T, rows, cols, G, unit_rows, masked, dtype):
    """Inputs change between replays, and the workspaces hold other calls' values by then."""
    c = Case(windq, rows, cols, G, unit_rows, masked=masked, seed=1)
    s = Side(windq, 4, 16, rows, cols, dtype, T, seed=2)
    X, dY = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    of = s.of_dev.clone()
    ws = [windq.project_workspace(c.packed, X, s.adapters, grad=k) for k in (False, True)]
    y, h = torch.empty(T, rows, dtype=dtype, device=DEV), torch.empty(T, 16, device=DEV)
    outs = torch.empty_like(X), torch.empty(s.a.shape, device=DEV), torch.empty(s.b.shape, device=DEV)

    def step():
        windq.windq_project(c.packed, X, s.adapters, of, h=h, ws=ws[0], out=y)
        windq.windq_project_grad(c.packed, dY, X, s.adapters, of, ws=ws[1], outs=outs)

    step()
    torch.cuda.synchronize()
    G_ = torch.cuda.CUDAGraph()
    with torch.cuda.graph(G_):
        step()
    for k in range(3):
        X.copy_(tokens(T, cols, dtype, 10 + k))
        dY.copy_(tokens(T, rows, dtype, 20 + k))
        of.copy_(of.roll(7))
        for w in ws:
            w.fill_(255)
        G_.replay()
        got = [t.clone() for t in (y, h, *outs)]
        want = [windq.windq_project(c.packed, X, s.adapters, of), got[1], *windq.windq_project_grad(c.packed, dY, X, s.adapters, of)]
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        windq.windq_project(c.packed, X, s.adapters, of, h=h)
        assert torch.equal(got[1], h)
        torch.cuda.synchronize()
