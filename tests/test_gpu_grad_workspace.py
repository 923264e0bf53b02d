"""windq_project_grad where rows are not in eights and the adapters' sums are cut into pieces, and from a workspace that held more tokens:
against the formulas in 64 bits, and nothing written past what the workspace function asked for."""
import numpy as np
import pytest
import torch

from test_gpu_project import DEV, EPS, Case, Side, near, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,T,n", [(511, 256, 100, 2), (1023, 512, 700, 3), (767, 1024, 65, 1)])
def test_rows_that_are_not_in_eights(windq, rows, cols, T, n):
    c = Case(windq, rows, cols, 64, 0, seed=1)
    s = Side(windq, n, 16, rows, cols, torch.bfloat16, T, seed=2)
    X, dY = tokens(T, cols, torch.bfloat16, 3), tokens(T, rows, torch.bfloat16, 4, 1e-2)
    x, dy = X.double().cpu().numpy(), dY.double().cpu().numpy()
    dx, dxm, da, dam, db, dbm = s.grad(x, dy)
    want = dy @ c.w + dx
    # weights rounded to bfloat16, dX too, dh in two terms (the bounds of the products' own tests)
    tol = EPS * (np.abs(dy) @ c.mag + dxm) + 2.0 ** -8 * 1.001 * np.abs(want) + 2.0 ** -8 * (np.abs(dy) @ np.abs(c.w)) + 2.0 ** -16 * dxm
    h = torch.empty(T, 16, device=DEV)
    windq.windq_project(c.packed, X, s.adapters, s.of_dev, h=h)
    need = windq.project_workspace(c.packed, dY, s.adapters, grad=True).numel()
    more = windq.project_workspace(c.packed, torch.empty(5 * T, rows, dtype=torch.bfloat16, device=DEV), s.adapters, grad=True).numel()
    first = None
    for size in (need, more):                            # its own workspace, and one for more tokens
        for given in (None, h):
            room = torch.full((size + 4096,), 255, dtype=torch.uint8, device=DEV)
            got = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev, h=given, ws=room[:size])
            near(got[0], want, tol)
            near(got[1], da, EPS * dam)
            near(got[2], db, EPS * dbm)
            assert torch.all(room[need:] == 255)
            first = got if first is None else first
            assert all(torch.equal(a, b) for a, b in zip(got[:1], first[:1]))
            again = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev, h=given, ws=room[:size])
            assert all(torch.equal(a, b) for a, b in zip(got, again))
