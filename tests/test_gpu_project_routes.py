"""Every kernel that the adapter calls may take, by shapes that take it (which a test without a GPU holds them to), against the formulas in 64 bits.

Bounds are those of test_gpu_project: 16 x 2^-24 of the magnitudes that the instructions add, half a unit in the last place of a bfloat16 output,
2^-16 of products with an intermediate in two bfloat16 terms, 2^-8 of those with weights rounded to bfloat16."""
import numpy as np
import pytest
import torch

from test_gpu_project import DEV, EPS, Case, Side, near, tokens, y_tol

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# kernel (as mangled), type of X, type of W, tokens, rows, cols, chunk width, unit rows, adapters, ranks, mask
FORWARD = [
    ("project_few_kernelILi8ELi1ELi16ELb0E", BF, BF, 8, 320, 768, 128, 64, 3, 40, False),
    ("project_few_kernelILi6ELi1ELi16ELb0E", BF, F32, 1, 104, 960, 96, 0, 2, 16, False),
    ("project_few_kernelILi4ELi1ELi16ELb0E", BF, BF, 3, 72, 1280, 64, 0, 1, 8, False),
    ("project_few_kernelILi8ELi1ELi8ELb1E", BF, BF, 30, 264, 1024, 256, 0, 5, 24, False),
    ("project_few_kernelILi6ELi1ELi8ELb1E", BF, BF, 32, 96, 384, 96, 32, 4, 128, False),
    ("project_few_kernelILi4ELi2ELi8ELb1E", BF, F32, 50, 200, 640, 64, 0, 9, 32, False),
    ("project_few_kernelILi8ELi2ELi8ELb1E", BF, BF, 300, 256, 2176, 128, 0, 7, 48, False),
    ("project_few_kernelILi8ELi1ELi16ELb0E", BF, BF, 5, 96, 1536, 512, 0, 2, 16, False),          # 512 wide: whole rows of trits, 103 bytes each
    ("project_few_kernelILi8ELi1ELi8ELb1E", BF, F32, 20, 40, 2560, 512, 0, 2, 16, False),
    ("project_few_kernelILi8ELi2ELi8ELb1E", BF, BF, 100, 104, 1536, 512, 0, 3, 64, False),
    ("project_kernelItLi1ELb0E", BF, BF, 40, 100, 960, 160, 20, 3, 16, False),
    ("project_kernelItLi2ELb0E", BF, F32, 700, 250, 480, 32, 0, 6, 24, False),
    ("project_kernelItLi1ELb1E", BF, BF, 40, 256, 512, 128, 0, 3, 16, True),
    ("project_kernelItLi2ELb1E", BF, F32, 300, 512, 384, 96, 0, 3, 64, True),
    ("project_kernelIfLi1ELb0E", F32, F32, 70, 136, 640, 64, 0, 3, 40, False),
    ("project_kernelIfLi2ELb0E", F32, BF, 900, 201, 320, 160, 0, 5, 16, False),
    ("project_kernelIfLi1ELb1E", F32, BF, 9, 256, 512, 128, 0, 2, 8, True),
    ("project_kernelIfLi2ELb1E", F32, F32, 300, 512, 768, 256, 0, 3, 32, True),
    ("project_tiles_kernelItLi8E", BF, BF, 700, 1024, 512, 128, 0, 5, 64, False),
    ("project_tiles_kernelItLi8E", BF, F32, 1100, 1032, 896, 128, 0, 3, 128, False),                # fp32 skip weights; rows and tokens that end inside a tile
    ("project_tiles_kernelItLi8E", BF, BF, 650, 1280, 768, 128, 64, 0, 0, False),
    ("project_tiles_kernelItLi8E", BF, BF, 700, 1024, 768, 256, 0, 40, 16, False),                  # laid out anew, two k-blocks a chunk
    ("project_tiles_kernelItLi8E", BF, F32, 800, 960, 512, 512, 192, 2, 24, False),
    ("project_tiles_kernelItLi8E", BF, BF, 1601, 1024, 4352, 128, 128, 4, 32, False),               # 34 k-blocks
    ("project_tiles_kernelItLi6E", BF, BF, 700, 1024, 576, 96, 0, 3, 40, False),
    ("project_tiles_kernelItLi6E", BF, F32, 1100, 1000, 384, 192, 0, 6, 16, False),
    ("project_tiles_kernelItLi6E", BF, BF, 700, 1088, 576, 288, 64, 0, 0, False),
    ("project_tiles_kernelItLi4E", BF, BF, 700, 1024, 448, 64, 0, 3, 56, False),
    ("project_tiles_kernelItLi4E", BF, F32, 600, 1216, 640, 320, 64, 9, 16, False),
    ("project_tiles_kernelIfLi8E", F32, F32, 700, 1024, 512, 128, 0, 5, 64, False),
    ("project_tiles_kernelIfLi8E", F32, BF, 900, 712, 768, 256, 0, 3, 128, False),
    ("project_tiles_kernelIfLi8E", F32, F32, 1100, 576, 1408, 128, 64, 11, 24, False),
    ("project_tiles_kernelIfLi6E", F32, F32, 700, 1000, 576, 96, 0, 3, 40, False),
    ("project_tiles_kernelIfLi6E", F32, BF, 750, 768, 384, 192, 128, 0, 0, False),
    ("project_tiles_kernelIfLi4E", F32, F32, 700, 1024, 448, 64, 0, 3, 16, False),
    ("project_tiles_kernelIfLi4E", F32, BF, 640, 960, 640, 320, 64, 4, 32, False),
]

# kernels, type, type of W, tokens, rows, cols, chunk width, unit rows, adapters, ranks, mask
BACK = [
    (("dx_gemm_kernelILi4E", "outer_tiles_kernelILi4ELi8E", "shrink_kernelILi4E"), BF, BF, 2000, 136, 4096, 128, 0, 1, 64, False),
    (("dx_gemm_kernelILi4E", "outer_tiles_kernelILi4ELi8E", "shrink_kernelILi8E"), BF, F32, 1930, 264, 4160, 64, 0, 2, 128, False),
    (("dx_gemm_kernelILi4E", "outer_tiles_kernelILi2ELi4E"), BF, BF, 2500, 320, 4000, 160, 64, 7, 32, True),
    (("dx_gemm_kernelILi2E", "outer_tiles_kernelILi1ELi8E"), BF, BF, 2000, 136, 1024, 128, 0, 1, 16, False),
    (("dx_gemm_kernelILi2E", "outer_tiles_kernelILi3ELi8E", "dx_join_kernel", "shrink_kernelILi3E"), BF, F32, 600, 1088, 512, 64, 64, 1, 48, False),
    (("dx_gemm_kernelILi2E", "outer_tiles_kernelILi2ELi8E", "dx_join_kernel"), BF, BF, 1500, 2000, 384, 96, 0, 2, 24, False),
    (("dx_gemm_kernelILi2E", "outer_tiles_kernelILi4ELi4E", "shrink_kernelILi5E"), BF, BF, 513, 640, 520, 8, 0, 3, 80, False),
    (("dx_gemm_kernelILi2E", "outer_tiles_kernelILi4ELi4E", "shrink_kernelILi6E"), BF, BF, 300, 1023, 640, 128, 11, 5, 96, True),
    (("dx_gemm_kernelILi2E", "outer_tiles_kernelILi4ELi8E", "shrink_kernelILi7E"), BF, F32, 530, 777, 768, 256, 0, 1, 104, False),
    (("dx_f32_kernel", "dx_f32_join_kernel", "outer_kernel"), F32, F32, 300, 777, 768, 256, 0, 4, 104, False),
    (("dx_f32_kernel", "outer_kernel"), F32, BF, 1100, 200, 1032, 24, 40, 3, 16, True),
]


def case_of(windq, w_type, rows, cols, G, unit_rows, masked):
    return Case(windq, rows, cols, G, unit_rows, w_type, masked=masked, seed=rows + cols)


@pytest.mark.parametrize("kernel,x_type,w_type,T,rows,cols,G,unit_rows,n,rank,masked", FORWARD)
def test_the_way_there(windq, kernel, x_type, w_type, T, rows, cols, G, unit_rows, n, rank, masked):
    c = case_of(windq, w_type, rows, cols, G, unit_rows, masked)
    X = tokens(T, cols, x_type, T)
    x = X.double().cpu().numpy()
    want = x @ c.w.T
    near(windq.windq_project(c.packed, X), want, y_tol(c, x, x_type, want))
    if n == 0:
        return
    for order in ("mixed", "runs"):
        s = Side(windq, n, rank, rows, cols, x_type, T, seed=n, order=order)
        h, hm, side, sm = s.project(x)
        # a workspace for more tokens, full of NaN, and nothing written past what these tokens need
        need = windq.project_workspace(c.packed, X, s.adapters).numel()
        size = windq.project_workspace(c.packed, torch.empty(2 * T + 70, cols, dtype=x_type, device=DEV), s.adapters).numel()
        ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
        H = torch.full((T, rank), float("nan"), device=DEV)
        y = windq.windq_project(c.packed, X, s.adapters, s.of_dev, h=H, ws=ws)
        near(y, want + side, y_tol(c, x, x_type, want + side, sm))
        near(H, h, EPS * hm)
        assert torch.all(ws[need:] == 255)
        assert torch.equal(y, windq.windq_project(c.packed, X, s.adapters, s.of_dev))


@pytest.mark.parametrize("kernels,x_type,w_type,T,rows,cols,G,unit_rows,n,rank,masked", BACK)
def test_the_way_back(windq, kernels, x_type, w_type, T, rows, cols, G, unit_rows, n, rank, masked):
    c = case_of(windq, w_type, rows, cols, G, unit_rows, masked)
    X, dY = tokens(T, cols, x_type, T), tokens(T, rows, x_type, T + 1, 1e-2)
    x, dy = X.double().cpu().numpy(), dY.double().cpu().numpy()
    s = Side(windq, n, rank, rows, cols, x_type, T, seed=n)
    dx, dxm, da, dam, db, dbm = s.grad(x, dy)
    want = dy @ c.w + dx
    tol = EPS * (np.abs(dy) @ c.mag + dxm)
    if x_type == BF:
        tol += 2.0 ** -8 * 1.001 * np.abs(want) + 2.0 ** -8 * (np.abs(dy) @ np.abs(c.w)) + 2.0 ** -16 * dxm
    need = windq.project_workspace(c.packed, dY, s.adapters, grad=True).numel()
    size = windq.project_workspace(c.packed, torch.empty(2 * T + 70, rows, dtype=x_type, device=DEV), s.adapters, grad=True).numel()
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    got = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev, ws=ws)
    near(got[0], want, tol)
    near(got[1], da, EPS * dam)
    near(got[2], db, EPS * dbm)
    assert torch.all(ws[need:] == 255)
    again = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    if x_type == BF:                                     # rounded weights cost no more than their size suggests
        alone, want0 = windq.windq_project_grad(c.packed, dY)[0], dy @ c.w
        assert np.linalg.norm(alone.double().cpu().numpy() - want0) <= 4e-3 * np.linalg.norm(want0)
