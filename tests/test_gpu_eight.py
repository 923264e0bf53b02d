"""windq_tokens8, windq_project8 and windq_gated8 against the formulas in 64 bits.

Bounds.  The integer sums are exact, so that what a product is off comes from fp32 additions of terms whose magnitudes add up to M (alpha |sum f q| and |beta sum q| over the chunks,
no more than the sums of the magnitudes): 16 x 2^-24 M holds them, as roundings are relative to partial sums and of random sign.  bfloat16 outputs add half a unit in their
last place, at most 2^-8 |y|.  In H = act(G) U an error e of G comes out as 1.13 |U| e at most (no activation is steeper), one of U as |act(G)| e; the activation's own
arithmetic is some ten roundings of fp32, 16 x 2^-24 |H|, and where gelu_tanh or silu divide by 1 + e^z, of an exponent z that is off by 2^-23 |z|, that much of it."""
import numpy as np
import pytest
import torch

from test_gpu_project import Case, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 16 * 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def eight(x, width, G, kb):
    """The definition, one rounded fp32 operation after the other, on the CPU. -> codes [T, width], scale [T], sums [T, blocks in fours]"""
    x = x.float().cpu().numpy()
    T, cols = x.shape
    with np.errstate(all="ignore"):
        most = np.abs(x).max(1) if cols else np.zeros(T, np.float32)
        most = np.where(np.isnan(x).any(1), np.float32("nan"), most).astype(np.float32)
        sigma = (most / np.float32(127)).astype(np.float32)
        sigma = np.where(sigma < np.float32(2.0 ** -126), np.float32(0), sigma)
        fine = np.isfinite(most)
        inverse = np.where(fine & (sigma > 0), np.float32(1) / sigma, np.float32(0)).astype(np.float32)
        q = np.clip(np.rint((x * inverse[:, None]).astype(np.float32)), -127, 127)
    q = np.where(fine[:, None], q, 0).astype(np.int8)
    padded = width // (cols // G)
    codes = np.zeros((T, cols // G, padded), np.int8)
    codes[:, :, :G] = q.reshape(T, -1, G)
    codes = codes.reshape(T, width)
    sums = codes.reshape(T, -1, kb).astype(np.int32).sum(2)
    return codes, np.where(fine, sigma, np.float32("nan")), np.pad(sums, ((0, 0), (0, -sums.shape[1] % 4))), q


def block(G):
    steps = (G + 31) // 32
    parts = (steps + 3) // 4
    return 32 * -(-steps // parts)


def magnitudes(c):
    """|alpha f| + |beta| of every weight, as the products add them."""
    mag = np.abs(c.w).copy()
    sc, of = (x.double().cpu().numpy().reshape(-1, c.R_u, 1) for x in (c.scale, c.offset))
    nc = c.cols // c.G
    for u, a in enumerate(c.action.numpy()):
        if a == 0:
            continue
        here = np.s_[u // nc * c.R_u:(u // nc + 1) * c.R_u, u % nc * c.G:(u % nc + 1) * c.G]
        s, o = sc[u], of[u] if a < 5 else 0.0 * of[u]
        beta = {1: o + 128 * s, 5: -s, 6: -s}.get(int(a), o)
        mag[here] = np.abs(c.w[here] - beta) + np.abs(beta)
    return mag


def act(word, x):
    x = torch.from_numpy(x)
    y = x * torch.sigmoid(x) if word == "silu" else torch.nn.functional.gelu(x, approximate="tanh" if word == "gelu_tanh" else "none")
    return y.numpy()


def close(got, want, off, dtype):
    got = got.double().cpu().numpy()
    limit = off + (2.0 ** -8 * np.abs(want) if dtype == BF else 2.0 ** -24 * np.abs(want))
    worst = (np.abs(got - want) / np.maximum(limit, 1e-300)).max() if got.size else 0.0
    assert np.all(np.abs(got - want) <= limit), worst


SHAPES = [(64, 128, 64, 0, 1), (200, 480, 96, 40, 5), (72, 80, 8, 0, 33), (1000, 1056, 96, 0, 77), (128, 512, 256, 64, 64), (40, 1024, 512, 8, 65),
          (35, 800, 160, 0, 31), (96, 288, 72, 32, 130), (7, 256, 128, 1, 3), (320, 1280, 128, 64, 200), (513, 256, 64, 0, 257), (264, 384, 128, 88, 129),
          (72, 80, 8, 0, 333), (160, 320, 32, 32, 150), (300, 480, 160, 0, 390), (1000, 1056, 96, 0, 513), (2080, 768, 128, 0, 700), (576, 512, 512, 192, 1025),
          # tiles, by the rule for it: steps of 4, 3, 2 and 1, tile units, ragged rows, a last pair of one k-block
          (8192, 640, 128, 0, 700), (6000, 288, 96, 0, 900), (8192, 320, 64, 64, 650), (8200, 160, 32, 0, 640), (4160, 1024, 512, 32, 1200), (5000, 144, 72, 1000, 1090)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,cols,G", [(1, 8, 8), (3, 80, 8), (5, 1056, 96), (2, 4096, 128), (9, 11008, 128), (4, 72, 72), (2, 800, 160), (1, 512, 512), (300, 64, 64),
                                      (2, 33024, 8), (1, 131072, 64), (3, 2080, 160), (4, 5120, 256), (2, 14400, 96)])
def test_tokens8_is_the_definition_bit_for_bit(windq, dtype, T, cols, G):
    x = tokens(T, cols, dtype, 3)
    x[:, ::7] *= 6
    if T > 2:
        x[1] = 0.0
        x[2, 5] = float("inf") if dtype == BF else float("nan")
    if T > 4:
        x[3] = 1e-38                                        # its scale would be below the smallest normal fp32
        x[4, :] = 0.0
        x[4, 3] = -1.0
    t = windq.windq_tokens8(x, G)
    codes, scale, sums, _ = eight(x, t.codes.shape[1], G, block(G))
    assert np.array_equal(t.codes.cpu().numpy(), codes)
    assert np.array_equal(t.scale.cpu().numpy(), scale, equal_nan=True)
    assert np.array_equal(t.sums.cpu().numpy(), sums)


def test_tokens8_reads_strided_rows_and_ties_go_to_even(windq):
    whole = tokens(6, 512, BF, 4)
    x = whole[1:5:2, 128:384]                              # a leading dimension of two rows
    t = windq.windq_tokens8(x, 64)
    assert np.array_equal(t.codes.cpu().numpy(), eight(x, 256, 64, 64)[0])
    y = torch.zeros(1, 64, device=DEV)
    y[0, :6] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5])
    assert windq.windq_tokens8(y, 64).codes[0, :6].tolist() == [127, 0, 2, 2, 0, -2]


def products(windq, shape, w_dtype, seed=0, pair=False, only=None):
    rows, cols, G, unit_rows, T = shape
    cs = [Case(windq, rows, cols, G, unit_rows, w_dtype, seed=seed + k, only=only) for k in range(2 if pair else 1)]
    x = tokens(T, cols, BF, seed + 5)
    t = windq.windq_tokens8(x, G)
    q = eight(x, t.codes.shape[1], G, block(G))[3].astype(float)
    sigma = t.scale.double().cpu().numpy()[:, None]
    want = [sigma * (q @ c.w.T) for c in cs]
    off = [EPS * sigma * (np.abs(q) @ magnitudes(c).T) for c in cs]
    return cs, t, want, off


@pytest.mark.parametrize("w_dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_project8(windq, shape, w_dtype):
    (c,), t, (want,), (off,) = products(windq, shape, w_dtype)
    s = windq.Serving(c.packed)
    for dtype in (BF, F32):
        y = windq.windq_project8(s, t, dtype)
        close(y, want, off, dtype)
        assert torch.equal(y, windq.windq_project8(s, t, dtype))


@pytest.mark.parametrize("only", range(7))
@pytest.mark.parametrize("T", [1, 40, 300])
def test_project8_of_one_treatment(windq, only, T):
    (c,), t, (want,), (off,) = products(windq, (256, 640, 128, 0, T), BF, seed=only, only=only)
    close(windq.windq_project8(windq.Serving(c.packed), t, F32), want, off, F32)


@pytest.mark.parametrize("word", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gated8(windq, shape, word):
    w_dtype = F32 if shape[0] % 5 == 0 else BF
    cs, t, (g, u), (go, uo) = products(windq, shape, w_dtype, pair=True)
    plans = [windq.Serving(c.packed) for c in cs]
    a = act(word, g)
    want = a * u
    off = 1.13 * np.abs(u) * go + np.abs(a) * uo + 1.13 * go * uo + EPS * np.abs(want) * (1 + np.abs(g) + np.abs(g) ** 3 / 8)
    for dtype in (BF, F32):
        close(windq.windq_gated8(*plans, t, word, dtype), want, off, dtype)
