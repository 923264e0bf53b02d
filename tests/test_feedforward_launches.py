"""What the feed-forward calls launch: the host code alone, without a GPU."""
import ctypes

from host_launches import AT, recorder  # noqa: F401
from paper_2605_26660_amd import binding


def gated(recorder, shape, dtype=binding.WINDQ_BF16, w_dtype=None, mask=False, codes_bytes=1 << 30):
    """One call of windq_gated with made-up addresses. -> (status, the launches' names)"""
    B, L, ref = binding, recorder.lib, ctypes.byref
    rows, cols, G, unit_rows, T = shape
    W = B.windq_mat(AT, dtype if w_dtype is None else w_dtype, 0, rows, cols, cols)
    X = B.windq_mat(AT, dtype, 0, T, cols, cols)
    P = B.windq_packed(ctypes.pointer(W), AT if mask else None, AT, AT, AT, codes_bytes, AT, AT, G, 0, unit_rows)
    need = L.windq_gated_workspace_bytes(0, dtype, T, rows, cols, G)
    L.recorded_clear()
    status = L.windq_gated(ref(P), ref(P), ref(X), 0, AT, rows, AT, AT, rows, AT, need, None)
    return status, " ".join(x.name for x in recorder.launches())


def test_the_routes_tests_take_the_routes_they_name(recorder):
    """The shapes that are compared with 64 bits on the GPU, kernel by kernel: a rule that moves one of them to another kernel shows here."""
    import test_gpu_feedforward_routes as R

    for kernels, shape in R.HALVES + R.EXACT:
        status, names = gated(recorder, shape)
        assert status == 0 and all(k in names for k in kernels), (kernels, shape, names)


def gated_grad(recorder, shape, masked=False, dtype=binding.WINDQ_BF16):
    """One call of windq_gated_grad with made-up addresses. -> (status, the launches' names)"""
    B, L, ref = binding, recorder.lib, ctypes.byref
    rows, cols, G, unit_rows, T = shape
    W, dH = B.windq_mat(AT, dtype, 0, rows, cols, cols), B.windq_mat(AT, dtype, 0, T, rows, rows)
    P = B.windq_packed(ctypes.pointer(W), AT if masked else None, AT, AT, AT, 1 << 30, AT, AT, G, 0, unit_rows)
    need = L.windq_gated_workspace_bytes(1, dtype, T, rows, cols, G)
    L.recorded_clear()
    status = L.windq_gated_grad(ref(P), ref(P), ref(dH), AT, AT, rows, 0, AT, cols, AT, AT, rows, AT, need, None)
    return status, " ".join(x.name for x in recorder.launches())


def test_the_ways_back_take_the_routes_they_name(recorder):
    import test_gpu_feedforward_range as R

    for kernels, other, shape, masked in R.BACK:
        status, names = gated_grad(recorder, shape, masked)
        assert status == 0 and all(k in names for k in kernels) and other not in names, (kernels, shape, names)


def test_few_tokens_of_as_many_rows_as_the_header_allows(recorder):
    """A launch holds fewer than 2^32 threads: more rows go in several, none are refused."""
    for dtype in (binding.WINDQ_BF16, binding.WINDQ_F32):
        for shape in ((1 << 27, 64, 64, 0, 1), ((1 << 27) + 16, 64, 64, 0, 15), ((1 << 31) - 512, 64, 64, 0, 1), ((1 << 26) + 64, 64, 64, 0, 31), ((1 << 25) - 512, 64, 64, 32, 63)):
            status, _ = gated(recorder, shape, dtype, codes_bytes=1 << 40)
            launches = recorder.launches()
            assert status == 0 and all(0 < x.grid * x.block < 1 << 32 for x in launches), (dtype, shape, status, launches)
            rows, T = shape[0], shape[4]
            few = [x.grid for x in launches if "pair_few_kernel" in x.name]
            if few:
                assert sum(few) == -(-rows // 16) * -(-T // 16), (dtype, shape)
            mine = [x.grid for x in launches if "project_few_kernel" in x.name]
            if mine:
                assert sum(mine) == -(-rows // 32) * -(-T // (32 if T <= 32 else 64)), (dtype, shape)
            assert few or mine or "project_kernel" in launches[-1].name


def test_windq_project_of_as_many_rows_as_the_header_allows(recorder):
    for T, rows in ((1, 1 << 27), (8, (1 << 27) + 32), (1, (1 << 31) - 512), (31, (1 << 26) + 64), (63, (1 << 25) - 512)):
        status, _, _ = recorder.product(False, T, rows, 64, 64)
        launches = recorder.launches()
        assert status == 0 and all(0 < x.grid * x.block < 1 << 32 for x in launches), (T, rows, status)
        mine = [x.grid for x in launches if "project_few_kernel" in x.name]
        assert sum(mine) == -(-rows // 32) * -(-T // (32 if T <= 32 else 64)), (T, rows)
