"""What windq_project, windq_project_grad and windq_adamw launch, and what of the workspace they hand to it: the host code alone, without a GPU."""
import ctypes
import random

from host_launches import AT, recorder  # noqa: F401
from paper_2605_26660_amd import binding


def apart(regions, at, need):
    """The regions lie in the workspace and none reaches into another."""
    ends = sorted(regions)
    return all(at <= a <= b <= at + need for a, b in ends) and all(x[1] <= y[0] for x, y in zip(ends, ends[1:]))


def test_pieces_of_the_adapters_sums_stay_in_their_own_part_of_the_workspace(recorder):
    """Pieces are as many as the width allows, and dY's width is that of its rows in eights."""
    rng = random.Random(1)
    shapes = [(511, 256, 100, 2), (1023, 512, 700, 3), (4095, 4088, 64, 1)]
    for k in range(2, 33):
        shapes += [(256 * k - rng.randint(0, 9), 8 * rng.randint(1, 32 * k), rng.choice([1, 65, 100, 700, 3000]), rng.choice([1, 2, 5, 40])) for _ in range(6)]
    for rows, cols, T, n in shapes:
        for h in (False, True):
            status, at, need = recorder.product(True, T, rows, cols, 8, n=n, rank=16, h=h)
            assert status == 0
            regions = recorder.regions()
            assert len(regions) == (3 if h else 4) and apart(regions, at, need), (rows, cols, T, n, h)
            status, at, need = recorder.product(False, T, rows, cols, 8, n=n, rank=16, h=h)
            assert status == 0 and apart(recorder.regions(), at, need)


def names(recorder):
    return " ".join(x.name for x in recorder.launches())


def test_codes_are_read_in_whole_pieces_only_where_the_stream_has_them_whole(recorder):
    """The kernel for few tokens reads a unit's codes 16 bytes at a time, and units start on 16: a stream of whole pieces holds the last one whole."""
    for rows, G in ((8, 64), (40, 128), (24, 384)):
        for T in (1, 40):
            status, _, _ = recorder.product(False, T, rows, 4 * G, G, codes_bytes=4096)
            assert status == 0 and "project_few_kernel" in names(recorder)
            for left in (1, 8, 15):                          # 8 rows of 1.58 bits at G = 64 are 104 bytes
                status, _, _ = recorder.product(False, T, rows, 4 * G, G, codes_bytes=4096 + left)
                assert status == 0 and "project_few_kernel" not in names(recorder) and "project_kernel" in names(recorder)


def test_sizes_that_no_card_holds_are_refused_instead_of_wrapping_round(recorder):
    """Bytes of a workspace are counted in 64 bits: what would pass them, or a side that a kernel's 32-bit index would, is out of range."""
    L, F, B = recorder.lib, 0, 1
    side = (1 << 31) - 512
    for grad, dtype, T, rows, cols, G, n, rank in ((0, F, (1 << 31) - 1, 1, 1 << 31, 8, 0, 0), (0, F, 1 << 30, 1, side, 8, 0, 0), (1, F, 8, 8, side + 8, 8, 0, 0),
                                                   (1, B, 1, side + 8, 8, 8, 0, 0), (0, F, 1, 1, 1 << 31, 512, 0, 0), (1, B, 10, side, side, 8, (1 << 20), 128),
                                                   (1, B, 1000, side, 8, 8, 0, 0), (1, B, 1000, 8, side, 8, 0, 0), (0, B, 10, 64, 64, 64, (1 << 20) + 1, 8),
                                                   (0, B, 10, 1 << 24, 1 << 24, 64, 0, 0), (0, B, 10, 64, 1 << 24, 64, 1 << 20, 128)):
        assert L.windq_project_workspace_bytes(grad, dtype, T, rows, cols, G, n, rank) == 0
        status, _, _ = recorder.product(grad, T, rows, cols, G, dtype=dtype, n=n, rank=rank)
        assert status == 2 and not recorder.launches()            # WINDQ_ESHAPE
    for grad in (0, 1):                                       # whatever comes out is what the parts add up to
        for dtype in (F, B):
            for T, rows, cols in ((1, 1 << 24, 1 << 12), (1 << 17, 1 << 13, 1 << 13), (100, 1 << 14, 1 << 20)):
                planes = 6 * T * cols if dtype == F and not grad else 2 * rows * cols if dtype == B and grad else 0
                assert planes <= L.windq_project_workspace_bytes(grad, dtype, T, rows, cols, 128, 0, 0) < 1 << 44


def test_no_launch_holds_as_many_threads_as_the_runtime_cuts_short(recorder):
    """A launch of 2^32 threads or more loses the rest without an error: work of that size goes in several, and no size is refused between them."""
    F, B = 0, 1
    for grad, dtype, T, rows, cols, G, n, rank, kernel, workgroups in (
            (0, F, 1 << 20, 8, 64, 64, 4, 128, "shrink_token_kernel", 1 << 25), (1, F, 1 << 20, 8, 64, 64, 4, 128, "shrink_token_kernel", 1 << 26),
            (0, F, (1 << 19) + 77, 16, 64, 64, 4, 128, "shrink_token_kernel", 32 * ((1 << 19) + 77)),
            (1, B, 500, 4096, 4096, 128, 200000, 8, "outer_tiles_kernel", 200000 * 64), (1, B, 500, 4096, 4096, 128, 200000, 8, "grad_prepare_kernel", 200000 * 129 + 64 * 16),
            (1, F, 500, 4096, 4096, 128, 1000000, 8, "outer_kernel", 1000000 * 32), (1, B, 500, 64, 64, 64, 1 << 20, 128, "join_kernel", None),
            (0, B, (1 << 28) - 1, 8, 64, 64, 0, 0, "project_kernel", 1 << 23), (0, B, (1 << 25) - 1, 64, 640, 64, 0, 0, "tiles_prepare_kernel", 10 + 10 * (1 << 21)),
            (1, F, (1 << 28) - 1, 8, 8, 8, 0, 0, "dx_f32_kernel", 1 << 22), (1, B, (1 << 28) - 1, 1, 8, 8, 0, 0, "align_kernel", 1 << 26),
            (0, B, (1 << 28) - 1, 8, 64, 64, 1, 128, "join_kernel", None), (0, B, (1 << 28) - 1, 8, 64, 64, 4, 8, "shrink_kernel", None)):
        status, _, _ = recorder.product(grad, T, rows, cols, G, dtype=dtype, n=n, rank=rank)
        all_ = recorder.launches()
        assert status == 0 and all(x.grid * x.block < 1 << 32 for x in all_), (kernel, status)
        mine = [x.grid for x in all_ if kernel + "I" in x.name or kernel + "E" in x.name]
        assert mine and (workgroups is None or sum(mine) == workgroups), (kernel, mine)


def test_a_plan_of_skip_units_alone_needs_no_codes(recorder):
    """As for the other calls on a packed plan: no codes are given where there are none."""
    L, B = recorder.lib, binding
    W, X = B.windq_mat(AT, 1, 0, 64, 128, 128), B.windq_mat(AT, 1, 0, 9, 128, 128)
    for codes, codes_bytes, want in ((None, 0, 0), (None, 16, 1), (AT, 0, 0)):
        P = B.windq_packed(ctypes.pointer(W), None, AT, AT, codes, codes_bytes, AT, AT, 64, 0, 0)
        assert L.windq_project(ctypes.byref(P), ctypes.byref(X), None, None, AT, 64, None, AT, 1 << 30, None) == want


def test_the_routes_tests_take_the_routes_they_name(recorder):
    """The shapes that are compared with 64 bits on the GPU, kernel by kernel: a rule that moves one of them to another kernel shows here."""
    import torch

    import test_gpu_project_routes as R

    code = {torch.bfloat16: 1, torch.float32: 0}
    for kernel, x_type, w_type, T, rows, cols, G, unit_rows, n, rank, masked in R.FORWARD:
        for adapters in {0, n}:
            status, _, _ = recorder.product(False, T, rows, cols, G, unit_rows, code[x_type], adapters, rank if adapters else 0, masked, code[w_type], codes_bytes=1 << 20)
            assert status == 0 and kernel in names(recorder), (kernel, names(recorder))
    for kernels, x_type, w_type, T, rows, cols, G, unit_rows, n, rank, masked in R.BACK:
        status, _, _ = recorder.product(True, T, rows, cols, G, unit_rows, code[x_type], n, rank, masked, code[w_type], codes_bytes=1 << 20)
        assert status == 0 and all(k in names(recorder) for k in kernels), (kernels, names(recorder))
