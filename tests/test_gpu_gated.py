"""windq_gated and windq_gated_grad against the formulas in 64 bits, and the gradients against differences of them.

Bounds.  G and U are products as windq_project has them: 16 x 2^-24 of the sum of the magnitudes that are added; a bfloat16 output adds 2^-8 of its value.  Where many bfloat16
tokens go through weights in half precision, every weight is off by half a step of 2^-10 (2^-11 of it) at most, or, below 2^-14 of eight rows' largest times a power
of two (2^14 at least), half a step of 2^-24: 2^-39 of the largest; a token's values by 2^-39 of its largest.  In H an error e of G
comes out as 1.13 |U| e at most, one of U as |act(G)| e; the activation and its slope are some ten fp32 roundings of terms no larger than (1 + |G|) and, where an
exponent z of e^z is rounded first, |z| of them more, |z| < 2 (|G| + |G|^3 / 20): 16 x 2^-24 (1 + |G| + |G|^3 / 8).
dX in bfloat16: dG, dU and the weights enter in half precision, half a step of 2^-11 each, every weight and every way of rounding, and below 2^-14 (of the largest of a token or
chunk times a power of two, which is 2^14 at least) half a step of 2^-25; fp32 calls round neither."""
import numpy as np
import pytest
import torch

from test_gpu_eight import act, close
from test_gpu_project import Case, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 16 * 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def slope(word, g):
    x = torch.from_numpy(g).requires_grad_()
    y = x * torch.sigmoid(x) if word == "silu" else torch.nn.functional.gelu(x, approximate="tanh" if word == "gelu_tanh" else "none")
    return torch.autograd.grad(y.sum(), x)[0].numpy()


def curve(g):
    return 1 + np.abs(g) + np.abs(g) ** 3 / 8


def pair(windq, shape, dtype, masked=False, w_dtype=None, seed=0):
    rows, cols, G, unit_rows, _ = shape
    return [Case(windq, rows, cols, G, unit_rows, dtype if w_dtype is None else w_dtype, masked=masked and k != 1, seed=seed + k) for k in range(2)]


def forward(cs, x, word, dtype):
    """(G, U, H) in 64 bits and how far each may be off before its own rounding."""
    x = x.double().cpu().numpy()
    g, u = (x @ c.w.T for c in cs)
    go, uo = (EPS * (np.abs(x) @ c.mag.T) for c in cs)
    if dtype == BF and x.shape[0] > 64:
        size = np.abs(x)
        halves = lambda c: size @ (2.0 ** -11 * np.abs(c.w) + 2.0 ** -38 * np.abs(c.w).max()).T + 2.0 ** -38 * size.max(1, keepdims=True) * np.abs(c.w).sum(1)  # noqa: E731
        go, uo = go + halves(cs[0]), uo + halves(cs[1])
    a = act(word, g)
    return (g, u, a * u), (go, uo, 1.13 * np.abs(u) * go + np.abs(a) * uo + 1.13 * go * uo + EPS * np.abs(u) * curve(g))


# few tokens as they lie, laid out; tiles of 128, 96 and 64 columns and of wider chunks; the general kernel; tile units, rows that end inside a tile
SHAPES = [(64, 128, 64, 0, 1), (256, 512, 128, 0, 7), (352, 768, 96, 32, 40), (256, 512, 256, 0, 64), (200, 480, 96, 40, 5), (72, 80, 8, 0, 33), (1000, 1056, 96, 0, 77),
          (35, 800, 160, 0, 31), (1096, 512, 128, 0, 1100), (2048, 384, 64, 64, 700), (704, 768, 256, 64, 1300), (1032, 480, 96, 0, 1210)]


@pytest.mark.parametrize("word", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_gated(windq, shape, dtype, word):
    cs = pair(windq, shape, dtype, seed=shape[0] % 7)
    x = tokens(shape[4], shape[1], dtype, 4, 2.0)
    save = torch.full((2, shape[4], shape[0] + 3), 7.0, dtype=dtype, device=DEV)
    h = windq.windq_gated(cs[0].packed, cs[1].packed, x, word, save=(save[0, :, :-3], save[1, :, :-3]))
    want, off = forward(cs, x, word, dtype)
    for got, w, o in zip((save[0, :, :-3], save[1, :, :-3], h), want, off):
        close(got, w, o, dtype)
    assert torch.all(save[:, :, -3:] == 7.0)
    out = torch.full((shape[4], shape[0] + 1), 5.0, dtype=dtype, device=DEV)          # rows on no alignment
    assert torch.equal(windq.windq_gated(cs[0].packed, cs[1].packed, x, word, out=out[:, :-1]), h) and torch.all(out[:, -1] == 5.0)


@pytest.mark.parametrize("dtype,w_dtype", [(BF, BF), (F32, BF), (BF, F32)])
@pytest.mark.parametrize("T", [3, 90, 600])
def test_gated_of_a_masked_and_an_unmasked_plan(windq, dtype, w_dtype, T):
    shape = (320, 512, 128, 64, T)
    cs = pair(windq, shape, dtype, masked=True, w_dtype=w_dtype)
    x = tokens(T, 512, dtype, 5)
    for order in (cs, cs[::-1]):
        want, off = forward(order, x, "silu", dtype)
        close(windq.windq_gated(order[0].packed, order[1].packed, x), want[2], off[2], dtype)


def backward(cs, dh, g, u, word, dtype):
    dh, g, u = (t.double().cpu().numpy() for t in (dh, g, u))
    dg, du = dh * u * slope(word, g), dh * act(word, g)
    dx = dg @ cs[0].w + du @ cs[1].w
    go, uo = EPS * np.abs(dh * u) * curve(g), EPS * np.abs(dh * g) * curve(g)
    w = [np.abs(c.w) for c in cs]
    part = lambda a, b: a @ w[0] + b @ w[1]  # noqa: E731
    xo = part(go, uo) + EPS * part(np.abs(dg), np.abs(du))
    if dtype == BF:
        xo = xo * (1 + 2.0 ** -10) + (2 * 2.0 ** -11 + 2.0 ** -22) * part(np.abs(dg), np.abs(du))
        most = np.maximum(np.abs(dh * u), np.abs(dh * g)).max(1, keepdims=True) * 1.13
        xo = xo + 2.0 ** -39 * most * (w[0].sum(0) + w[1].sum(0)) + 2.0 ** -39 * max(x.max() for x in w) * 4 * (np.abs(dg) + np.abs(du)).sum(1, keepdims=True)
    return (dx, dg, du), (xo, go, uo)


@pytest.mark.parametrize("word", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_gated_grad(windq, shape, dtype, word):
    rows, T = shape[0], shape[4]
    cs = pair(windq, shape, dtype, seed=shape[0] % 5)
    dh, g, u = tokens(T, rows, dtype, 6, 1e-3), tokens(T, rows, dtype, 7, 2.0), tokens(T, rows, dtype, 8, 1.5)
    packed = [c.packed for c in cs]
    got = windq.windq_gated_grad(*packed, dh, g, u, word)
    want, off = backward(cs, dh, g, u, word, dtype)
    for a, b, o in zip(got, want, off):
        close(a, b, o, dtype)
    # rows of nothing aligned, outputs between sentinels, one part alone: the same values
    pad = lambda t: torch.nn.functional.pad(t, (1, 2))[:, 1:-2]  # noqa: E731
    outs = [torch.full((t.shape[0], t.shape[1] + 3), 9.0, dtype=dtype, device=DEV) for t in got]
    windq.windq_gated_grad(*packed, pad(dh), pad(g), pad(u), word, outs=tuple(o[:, :-3] for o in outs))
    for o, t in zip(outs, got):
        assert torch.equal(o[:, :-3], t) and torch.all(o[:, -3:] == 9.0)
    alone = windq.windq_gated_grad(*packed, dh, g, u, word, want_dgu=False), windq.windq_gated_grad(*packed, dh, g, u, word, want_dx=False)
    assert torch.equal(alone[0][0], got[0]) and torch.equal(alone[1][1], got[1]) and torch.equal(alone[1][2], got[2]) and alone[1][0] is None


@pytest.mark.parametrize("word", ["silu", "gelu", "gelu_tanh"])
def test_gradients_against_differences_of_the_formula(windq, word):
    shape = (96, 256, 64, 0, 6)
    cs = pair(windq, shape, F32)
    x, dh = tokens(6, 256, F32, 9, 2.0), tokens(6, 96, F32, 10)
    g, u = (torch.empty(6, 96, device=DEV) for _ in range(2))
    windq.windq_gated(cs[0].packed, cs[1].packed, x, word, save=(g, u))
    dx = windq.windq_gated_grad(cs[0].packed, cs[1].packed, dh, g, u, word)[0].double().cpu().numpy()
    off = backward(cs, dh, g, u, word, F32)[1][0]
    x64, d = x.double().cpu().numpy(), dh.double().cpu().numpy()
    loss = lambda z: (act(word, z @ cs[0].w.T) * (z @ cs[1].w.T) * d).sum(1)  # noqa: E731
    step = 1e-5
    # G and U are rounded to fp32 on their way: 2^-24 of them, through slopes below 1.2 and second derivatives below 1.2
    size = np.abs(x64) @ np.abs(cs[0].w).T + np.abs(x64) @ np.abs(cs[1].w).T
    saved = 2 * EPS * ((np.abs(d) * size * (1 + size)) @ (np.abs(cs[0].w) + np.abs(cs[1].w)))
    for k in (0, 1, 63, 64, 200, 255):
        e = np.zeros(256)
        e[k] = step
        want = (loss(x64 + e) - loss(x64 - e)) / (2 * step)
        assert np.all(np.abs(dx[:, k] - want) <= off[:, k] + saved[:, k] + 1e-7 * np.abs(want) + 1e-8), k


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_step_as_it_would_be_trained_and_served(windq, dtype):
    """The block forward with what its way back needs, back, and the gate's adapters from dG; the served form agrees with the trained one."""
    shape = (512, 768, 128, 0, 96)
    cs = pair(windq, shape, dtype)
    packed = [c.packed for c in cs]
    x, dh = tokens(96, 768, dtype, 11), tokens(96, 512, dtype, 12, 1e-2)
    save = tuple(torch.empty(96, 512, dtype=dtype, device=DEV) for _ in range(2))
    h = windq.windq_gated(*packed, x, save=save)
    dx, dg, du = windq.windq_gated_grad(*packed, dh, *save)
    want, off = backward(cs, dh, *save, "silu", dtype)
    close(dx, want[0], off[0], dtype)
    # dG, dU through windq_project_grad: dX's parts, by another route
    parts = [windq.windq_project_grad(p, d)[0].double().cpu().numpy() for p, d in zip(packed, (dg, du))]
    rough = 4 * 2.0 ** -8 if dtype == BF else EPS
    assert np.all(np.abs(parts[0] + parts[1] - want[0]) <= off[0] + rough * (np.abs(want[1]) @ np.abs(cs[0].w) + np.abs(want[2]) @ np.abs(cs[1].w)))
    # served with 8-bit tokens: off by what rounding the tokens does
    t = windq.windq_tokens8(x, 128)
    served = windq.windq_gated8(*(windq.Serving(p) for p in packed), t, dtype=dtype).double().cpu().numpy()
    (g, u, hw), ho = forward(cs, x, "silu", dtype)
    half = 0.5001 * t.scale.double().cpu().numpy()[:, None]
    ge, ue = (half * np.abs(c.w).sum(1) + o for c, o in zip(cs, ho))
    a = np.abs(act("silu", g))
    assert np.all(np.abs(served - hw) <= (1.13 * np.abs(u) * ge + a * ue + 1.13 * ge * ue) * 1.01 + 2.0 ** -7 * np.abs(hw) + 1e-6)
    assert np.linalg.norm(served - h.double().cpu().numpy()) < 0.05 * np.linalg.norm(hw)
