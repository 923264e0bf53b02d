"""windq_gated's kernels by shapes that are held to take them, against the formulas in 64 bits (bounds as in the call's own tests): up to 16 tokens by 16 rows a
workgroup (8 and 16 wavefronts, chunks of one and of several k-blocks, tokens in every place), and tiles of 256 x 256 (fewer steps than buffers, edges of both sides)."""
import pytest
import torch

from test_gpu_eight import close
from test_gpu_gated import backward, forward, pair
from test_gpu_project import DEV, tokens

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# rows, cols, G, unit_rows, tokens; 8192 rows are 512 workgroups
FEW = [(8, 64, 64, 0, 1), (8200, 256, 128, 0, 1), (8224, 192, 64, 32, 16), (8256, 288, 96, 0, 15), (8, 288, 96, 0, 16), (24, 512, 256, 0, 9), (96, 1024, 512, 32, 2), (4096, 8320, 128, 0, 3),
       (40, 768, 384, 0, 16), (16, 9600, 96, 0, 5)]
# one round of 256 x 256 tiles where 256 x 128 are two
LARGE = [(2064, 64, 64, 0, 1930), (2056, 192, 64, 0, 2048), (2080, 384, 128, 32, 1793), (1001 * 2, 256, 128, 0, 2047)]


def check(windq, shape, x, w_dtype=BF, word="silu"):
    dtype = x.dtype
    cs = pair(windq, shape, dtype, w_dtype=w_dtype, seed=shape[0] % 7)
    T, rows = shape[4], shape[0]
    save = torch.full((2, T, rows + 8), 7.0, dtype=dtype, device=DEV)
    out = torch.full((T, rows + 1), 5.0, dtype=dtype, device=DEV)
    h = windq.windq_gated(cs[0].packed, cs[1].packed, x, word, save=(save[0, :, :-8], save[1, :, :-8]), out=out[:, :-1])
    want, off = forward(cs, x, word, dtype)
    for got, w, o in zip((save[0, :, :-8], save[1, :, :-8], h), want, off):
        close(got, w, o, dtype)
    assert torch.all(save[:, :, -8:] == 7.0) and torch.all(out[:, -1] == 5.0)
    # without what the way back needs, rows on 16 bytes: the same
    assert torch.equal(windq.windq_gated(cs[0].packed, cs[1].packed, x, word), h)
    return cs, h


@pytest.mark.parametrize("w_dtype", [BF, F32])
@pytest.mark.parametrize("word", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("shape", FEW)
def test_up_to_16_tokens(windq, shape, word, w_dtype):
    check(windq, shape, tokens(shape[4], shape[1], BF, 4, 2.0), w_dtype, word)


# up to 64 tokens, and more of them while they are one round of workgroups; past it the half precision product, narrow tiles first
@pytest.mark.parametrize("shape", [(8224, 256, 128, 32, 33), (352, 768, 96, 32, 64), (256, 512, 128, 0, 700), (40, 640, 64, 0, 1000), (8200, 256, 128, 0, 65), (8192, 128, 64, 0, 130),
                                   (4104, 512, 256, 0, 257), (16384, 64, 64, 0, 129)])
def test_tokens_between(windq, shape):
    check(windq, shape, tokens(shape[4], shape[1], BF, 4, 2.0))


# fp32 by 16 rows and 16 tokens a workgroup: the last ones not full, and tiles beyond
@pytest.mark.parametrize("w_dtype", [BF, F32])
@pytest.mark.parametrize("shape", FEW + [(1000, 384, 96, 0, 301), (264, 512, 256, 0, 130), (96, 192, 64, 32, 1000), (2048, 256, 128, 0, 600)])
def test_fp32(windq, shape, w_dtype):
    check(windq, shape, tokens(shape[4], shape[1], F32, 4, 2.0), w_dtype, "gelu")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("only", range(7))
@pytest.mark.parametrize("G", [64, 96, 128, 256])
def test_up_to_16_tokens_of_one_treatment(windq, only, G, dtype):
    """Every column has its place: unit vectors for tokens give the reconstruction's columns."""
    from test_gpu_project import Case
    rows, cols = 48, 4 * G
    cs = [Case(windq, rows, cols, G, 0, dtype, seed=k, only=only) for k in range(2)]
    for first in range(0, cols, 16):
        x = torch.zeros(16, cols, dtype=dtype, device=DEV)
        x[torch.arange(16), first + torch.arange(16)] = 1.0
        save = torch.empty(2, 16, rows, dtype=dtype, device=DEV)
        windq.windq_gated(cs[0].packed, cs[1].packed, x, save=(save[0], save[1]))
        (g, u, _), (go, uo, _) = forward(cs, x, "silu", dtype)
        close(save[0], g, go, dtype)
        close(save[1], u, uo, dtype)


@pytest.mark.parametrize("shape", [FEW[1], FEW[5], LARGE[2]])
def test_rows_of_tokens_further_apart_and_one_that_is_not_finite(windq, shape):
    rows, cols, T = shape[0], shape[1], shape[4]
    wide = torch.full((T, cols + 72), float("nan"), dtype=BF, device=DEV)
    x = wide[:, 8:8 + cols]
    x.copy_(tokens(T, cols, BF, 4, 2.0))
    cs, h = check(windq, shape, x)
    p = [c.packed for c in cs]
    assert torch.equal(windq.windq_gated(*p, x.contiguous()), h)
    for bad in (float("nan"), float("inf")):
        y = x.contiguous().clone()
        y[T // 2, cols - 1] = bad
        got = windq.windq_gated(*p, y)
        others = torch.arange(T, device=DEV) != T // 2
        assert torch.equal(got[others], h[others]) and not torch.isfinite(got[T // 2]).any()


@pytest.mark.parametrize("word", ["silu", "gelu"])
@pytest.mark.parametrize("shape", LARGE)
def test_large_tiles(windq, shape, word):
    check(windq, shape, tokens(shape[4], shape[1], BF, 4, 2.0), word=word)


@pytest.mark.parametrize("shape", [(256, 512, 128, 0, 400), (264, 480, 96, 24, 350)])
@pytest.mark.parametrize("only", range(7))
def test_half_precision_weights_of_one_treatment(windq, shape, only):
    """Both reconstructions in half precision, as they lie and turned."""
    from test_gpu_project import Case
    rows, cols, G, unit_rows, T = shape
    cs = [Case(windq, rows, cols, G, unit_rows, BF, seed=k, only=only) for k in range(2)]
    p = [c.packed for c in cs]
    x, dh, g, u = tokens(T, cols, BF, 1, 2.0), tokens(T, rows, BF, 2, 1e-3), tokens(T, rows, BF, 3, 2.0), tokens(T, rows, BF, 4)
    want, off = forward(cs, x, "silu", BF)
    close(windq.windq_gated(*p, x), want[2], off[2], BF)
    want, off = backward(cs, dh, g, u, "silu", BF)
    close(windq.windq_gated_grad(*p, dh, g, u)[0], want[0], off[0], BF)


@pytest.mark.parametrize("word", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [8, 1984, 2048, 2056, 4104, 6152, 8200, 12288, 12296])
def test_gradients_of_rows_kept_in_registers_and_read_twice(windq, rows, word):
    """One to six octets of a row a thread, and more; where rows lie on no alignment they are read twice: the same bits."""
    shape = (rows, 64, 64, 0, 3)
    cs = pair(windq, shape, BF, seed=rows % 7)
    p = [c.packed for c in cs]
    dh, g, u = tokens(3, rows, BF, 2, 1e-3), tokens(3, rows, BF, 3, 2.0), tokens(3, rows, BF, 4)
    got = windq.windq_gated_grad(*p, dh, g, u, word)
    want, off = backward(cs, dh, g, u, word, BF)
    for a, b, o in zip(got, want, off):
        close(a, b, o, BF)
    pad = lambda t: torch.nn.functional.pad(t, (1, 2))[:, 1:-2]  # noqa: E731
    for a, b in zip(windq.windq_gated_grad(*p, pad(dh), pad(g), pad(u), word), got):
        assert torch.equal(a, b)
    assert torch.equal(windq.windq_gated_grad(*p, dh, g, u, word, want_dgu=False)[0], got[0])
