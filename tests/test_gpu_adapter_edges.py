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
