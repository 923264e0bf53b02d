"""windq_gated's kernels for many tokens and for chunks and rows of every kind, by shapes that a test without a GPU holds to take them: what is not finite, malformed
or at both ends of the range, each treatment by itself, strides, graphs and streams, against 64 bits (bounds as in the calls' own tests) or bit for bit."""
import pytest
import torch

import test_gpu_feedforward_edges as E
from test_gpu_eight import close
from test_gpu_gated import backward, forward, pair
from test_gpu_gated_routes import check
from test_gpu_project import DEV, Case, tokens

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# kernels (as mangled), rows, cols, G, unit_rows, tokens: the reconstruction in half precision and its product, every treatment in each of the matrices
HALVES = [(("gated_halves_kernelILb1ELi4E", "dx_gemm_kernelILi2ELb1ELb1E"), (1096, 896, 128, 0, 700)),
          (("gated_halves_kernelILb1ELi4E", "dx_gemm_kernelILi2ELb1ELb1E"), (704, 768, 256, 64, 1300)),
          (("gated_halves_kernelILb1ELi3E", "dx_gemm_kernelILi2ELb1ELb1E"), (1032, 672, 96, 0, 700)),
          (("gated_halves_kernelILb1ELi2E", "dx_gemm_kernelILi2ELb1ELb1E"), (2048, 448, 64, 64, 700)),
          (("gated_halves_kernelILb1ELi0E", "dx_gemm_kernelILi2ELb1ELb1E"), (1096, 1120, 160, 0, 400)),
          (("gated_halves_kernelILb0ELi0E", "dx_gemm_kernelILi2ELb1ELb1E"), (1032, 896, 128, 24, 700)),
          (("gated_halves_kernelILb1ELi4E", "dx_gemm_kernelILi4ELb1ELb1E"), (2048, 896, 128, 0, 2048)),
          (("gated_halves_kernelILb1ELi4E", "pair_gemm_kernel"), (2080, 384, 128, 32, 2047)),
          (("gated_halves_kernelILb1ELi3E", "pair_gemm_kernel"), (2056, 672, 96, 0, 2047))]
# kernels that do not round weights, whatever the tokens: for few of them, and the general one
EXACT = [(("project_few_kernelILi6ELi2ELi8ELb1ELb1E",), (1000, 1056, 96, 0, 77)), (("project_few_kernelILi8ELi2ELi8ELb1ELb1E",), (256, 512, 128, 0, 700)),
         (("project_few_kernelILi4ELi2ELi8ELb1ELb1E",), (40, 640, 64, 0, 1000)), (("project_kernelItLi2ELb0ELb1E",), (1001, 512, 128, 0, 400)),
         (("project_kernelItLi2ELb0ELb1E",), (2002, 256, 128, 0, 2047)), (("project_kernelItLi1ELb0ELb1E",), (35, 800, 160, 0, 400))]
SHAPES = [shape for _, shape in HALVES]


@pytest.fixture(autouse=True)
def memory():
    """What a test took goes back, for the tests behind it."""
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("word", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("shape", SHAPES)
def test_values(windq, shape, word):
    check(windq, shape, tokens(shape[4], shape[1], BF, 4, 2.0), word=word)


@pytest.mark.parametrize("w_dtype", [BF, F32])
@pytest.mark.parametrize("shape", [shape for _, shape in EXACT])
def test_values_where_no_weight_is_rounded(windq, shape, w_dtype):
    """As many tokens as others have in half precision, without the room that it takes."""
    cs = pair(windq, shape, BF, w_dtype=w_dtype, seed=shape[0] % 7)
    x = tokens(shape[4], shape[1], BF, 4, 2.0)
    save = torch.empty(2, shape[4], shape[0], dtype=BF, device=DEV)
    h = windq.windq_gated(cs[0].packed, cs[1].packed, x, save=(save[0], save[1]))
    want, off = forward(cs, x, "silu", F32)
    for got, w, o in zip((save[0], save[1], h), want, off):
        close(got, w, o, BF)


@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** -100])
@pytest.mark.parametrize("shape", SHAPES)
def test_tokens_at_both_ends_of_the_range(windq, shape, size):
    rows, cols, _, _, T = shape
    cs = pair(windq, shape, BF)
    x = tokens(T, cols, BF, 1)
    x[::3] *= size
    save = torch.empty(2, T, rows, dtype=BF, device=DEV)
    windq.windq_gated(*(c.packed for c in cs), x, save=(save[0], save[1]))
    want, off = forward(cs, x, "silu", BF)
    close(save[0], want[0], off[0] + 2.0 ** -133, BF)      # bfloat16's last place below the normal numbers
    close(save[1], want[1], off[1] + 2.0 ** -133, BF)


@pytest.mark.parametrize("only", range(7))
@pytest.mark.parametrize("shape", [SHAPES[k] for k in (0, 1, 2, 3, 4, 7)])
def test_one_treatment(windq, shape, only):
    """The reconstruction as it lies, in units of whole blocks of rows, and the product behind it."""
    rows, cols, G, unit_rows, T = shape
    cs = [Case(windq, rows, cols, G, unit_rows, BF, seed=k, only=only) for k in range(2)]
    x = tokens(T, cols, BF, 1, 2.0)
    want, off = forward(cs, x, "silu", BF)
    close(windq.windq_gated(*(c.packed for c in cs), x), want[2], off[2], BF)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_token_that_is_not_finite_is_nobody_elses(windq, shape, bad):
    E.test_a_token_that_is_not_finite_is_nobody_elses(windq, (*shape, BF), bad)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("what", ["scale", "offset", "skip"])
def test_a_weight_that_is_not_finite_is_its_rows_and_columns(windq, shape, what):
    for second in (False, True):
        E.test_a_weight_that_is_not_finite_is_its_rows_and_columns(windq, (*shape, BF), what, second)


@pytest.mark.parametrize("shape", SHAPES)
def test_malformed_entries_count_as_skip(windq, shape):
    E.test_malformed_entries_count_as_skip(windq, (*shape, BF))


@pytest.mark.parametrize("shape", SHAPES)
def test_captured_and_replayed(windq, shape):
    E.test_captured_and_replayed(windq, (*shape, BF))


@pytest.mark.parametrize("shape", SHAPES)
def test_rows_further_apart(windq, shape):
    """X, H, G and U as windows: the bits of the same values in close rows, what lies between left as it was."""
    rows, cols, _, _, T = shape
    cs = pair(windq, shape, BF)
    p = [c.packed for c in cs]
    wide = torch.full((T, cols + 72), float("nan"), dtype=BF, device=DEV)
    x = wide[:, 8:8 + cols].copy_(tokens(T, cols, BF, 4))
    plain = torch.empty(2, T, rows, dtype=BF, device=DEV)
    h = windq.windq_gated(*p, x.contiguous(), save=(plain[0], plain[1]))
    out, save = torch.full((T, rows + 3), 5.0, dtype=BF, device=DEV), torch.full((2, T, rows + 5), 7.0, dtype=BF, device=DEV)
    windq.windq_gated(*p, x, save=(save[0, :, 2:-3], save[1, :, 2:-3]), out=out[:, 1:-2])
    assert torch.equal(out[:, 1:-2], h) and torch.equal(save[:, :, 2:-3], plain)
    assert torch.all(out[:, 0] == 5.0) and torch.all(out[:, -2:] == 5.0) and torch.all(save[:, :, :2] == 7.0) and torch.all(save[:, :, -3:] == 7.0)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[7]])
def test_on_a_stream_of_its_own(windq, shape):
    """The call waits for nothing but its stream, whose earlier work it sees."""
    rows, cols, _, _, T = shape
    cs = pair(windq, shape, BF)
    p = [c.packed for c in cs]
    x, dh = tokens(T, cols, BF, 1), tokens(T, rows, BF, 2)
    save = torch.empty(2, T, rows, dtype=BF, device=DEV)

    def run(x, dh):
        h = windq.windq_gated(*p, x, save=(save[0], save[1]))
        return h, *windq.windq_gated_grad(*p, dh, save[0], save[1])

    want = [a.clone() for a in run(x, dh)]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        big = torch.ones(1 << 28, device=DEV)
        for _ in range(8):
            big.mul_(1.0)
        late_x, late_dh = torch.zeros_like(x), torch.zeros_like(dh)
        late_x.copy_(x), late_dh.copy_(dh)
        got = run(late_x, late_dh)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("word", ["silu", "gelu"])
@pytest.mark.parametrize("shape", [SHAPES[k] for k in (0, 2, 3, 5, 8)])
def test_there_and_back(windq, shape, word):
    rows, cols, _, _, T = shape
    cs = pair(windq, shape, BF, seed=3)
    p = [c.packed for c in cs]
    x, dh = tokens(T, cols, BF, 1, 2.0), tokens(T, rows, BF, 2, 1e-3)
    save = torch.empty(2, T, rows, dtype=BF, device=DEV)
    windq.windq_gated(*p, x, word, save=(save[0], save[1]))
    want, off = backward(cs, dh, save[0], save[1], word, BF)
    for a, b, o in zip(windq.windq_gated_grad(*p, dh, save[0], save[1], word), want, off):
        close(a, b, o, BF)


@pytest.mark.parametrize("T", [1, 15])                      # 2^31 - 1 tokens x rows at most
def test_more_rows_than_one_launch_holds(windq, T):
    """Rows on both sides of where one launch ends and the next begins, the last ones, and all of them written: windq_gated and windq_project of few tokens."""
    rows, cols = (1 << 27) + 48, 64
    g = torch.Generator(device=DEV).manual_seed(T)
    W = torch.empty(rows, cols, dtype=BF, device=DEV)       # no unit stays as it is: never read
    action = torch.full((1,), 6, dtype=torch.uint8, device=DEV)
    off = torch.tensor([0, rows * 8], dtype=torch.int64, device=DEV)
    plans, parts = [], []
    for _ in range(2):
        codes = torch.randint(0, 256, (rows * 8,), generator=g, device=DEV, dtype=torch.uint8)
        scale = torch.rand(rows, generator=g, device=DEV) + 0.5
        plans.append(windq.Packed(W, cols, 0, action, off, codes, scale, torch.zeros(rows, device=DEV)))
        parts.append((codes.view(rows, 8), scale))
    x = tokens(T, cols, BF, 3)
    h = torch.full((T, rows), float("nan"), dtype=BF, device=DEV)
    windq.windq_gated(*plans, x, out=h)
    y = windq.windq_project(plans[0], x, out=torch.full((T, rows), float("nan"), dtype=BF, device=DEV))
    assert all(torch.isfinite(t[:, r:r + (1 << 24)]).all() for t in (h, y) for r in range(0, rows, 1 << 24))
    edges = [0xffffffff // threads * piece for threads in (512, 1024) for piece in (16, 32)]
    for at in [0, rows - 4096] + [e - 2048 for e in edges if e < rows]:
        here = slice(at, at + 4096)
        ref, off64 = [], []
        for codes, scale in parts:
            bits = (codes[here, :, None] >> torch.arange(8, device=DEV)) & 1
            w = ((2.0 * bits.reshape(-1, cols) - 1) * scale[here, None]).double().cpu().numpy()
            ref.append(x.double().cpu().numpy() @ w.T)
            off64.append(16 * 2.0 ** -24 * (abs(x.double().cpu().numpy()) @ abs(w).T))
        close(y[:, here], ref[0], off64[0], BF)
        a = E.act("silu", ref[0])
        close(h[:, here], a * ref[1], 1.13 * abs(ref[1]) * off64[0] + abs(a) * off64[1] + 1.13 * off64[0] * off64[1] + 16 * 2.0 ** -24 * abs(ref[1]) * (1 + abs(ref[0])), BF)
