"""Edges of the feed-forward calls, against the formulas in 64 bits (bounds as in the calls' own tests) or bit for bit against what may not differ."""
import numpy as np
import pytest
import torch

from test_gpu_eight import act, block, close, eight, magnitudes, products
from test_gpu_gated import backward, forward, pair, slope
from test_gpu_project import DEV, Case, tokens

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 16 * 2.0 ** -24

# windq_gated, windq_gated_grad: few bfloat16 tokens; the general kernel; tiles (fp32); halves by known units, by small units, by many chunks; halves' fallbacks
GATED = [(256, 512, 128, 0, 7, BF), (256, 512, 128, 0, 7, F32), (100, 256, 128, 0, 90, BF), (1096, 512, 128, 0, 300, BF), (1096, 512, 128, 0, 700, F32), (256, 512, 128, 0, 400, BF),
         (72, 256, 64, 8, 321, BF), (64, 4160, 8, 0, 330, BF), (35, 800, 160, 0, 400, BF), (1001, 512, 128, 0, 400, BF)]
# 8-bit tokens: few by one and by two fragments, tiles (by rounds of workgroups), fp32 weights among them
EIGHT = [(256, 512, 128, 0, 5, BF), (96, 288, 72, 32, 60, F32), (8192, 640, 128, 0, 700, BF), (4160, 1024, 512, 32, 1200, F32)]


@pytest.fixture(autouse=True)
def memory():
    """What a test took goes back, for the tests behind it."""
    yield
    torch.cuda.empty_cache()


def finite(x):
    return torch.isfinite(x)


@pytest.mark.parametrize("word", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_activations_and_slopes_far_from_zero(windq, word, dtype):
    """Where e^x or x^2 pass fp32: act(g) is g or 0 there, its slope 1 or 0."""
    cs = pair(windq, (256, 64, 64, 0, 1), dtype)
    some = torch.tensor([20.0, 40.0, 87.0, 88.5, 89.0, 104.0, 128.0, 200.0, 1e4, 1e10, 1.9e19, 1e20, 1e30, 3.3e38])
    g = torch.cat([some, -some, torch.zeros(228)])[None].to(dtype).to(DEV)
    dh, u = torch.ones(1, 256, dtype=dtype, device=DEV), torch.full((1, 256), 0.5, dtype=dtype, device=DEV)
    _, dg, du = windq.windq_gated_grad(*(c.packed for c in cs), dh, g, u, word)
    g64 = g.double().cpu().numpy()
    step = np.where(np.abs(g64) < 19, slope(word, g64), (g64 > 0) * 1.0)                    # 20 e^-20 < 2^-24 from there on
    close(dg, 0.5 * step, EPS * np.ones_like(g64), dtype)
    value = np.where(np.abs(g64) < 19, act(word, g64), np.maximum(g64, 0))
    close(du, value, EPS * np.ones_like(g64), dtype)


@pytest.mark.parametrize("size", [2.0 ** 118, 2.0 ** -118])
def test_gradients_at_both_ends_of_the_range(windq, size):
    """What powers of two scale on its way through half precision: results are in range where a token's power alone is not."""
    shape = (64, 256, 64, 0, 5)
    cs = pair(windq, shape, BF)
    dh, g, u = tokens(5, 64, BF, 1, size), tokens(5, 64, BF, 2), tokens(5, 64, BF, 3)
    got = windq.windq_gated_grad(*(c.packed for c in cs), dh, g, u)
    want, off = backward(cs, dh, g, u, "silu", BF)
    assert np.abs(want[0]).max() < 3e38
    for a, b, o in zip(got, want, off):
        close(a, b, o + 2.0 ** -133, BF)                   # bfloat16's last place below the normal numbers


def test_gradients_of_products_past_the_range(windq):
    """dH G is no fp32 number where dH act(G) is one."""
    cs = pair(windq, (64, 256, 64, 0, 5), BF)
    dh, g, u = tokens(5, 64, BF, 1), tokens(5, 64, BF, 2), tokens(5, 64, BF, 3)
    dh[1, 5], g[1, 5], u[1, 5] = 2.0 ** 126, -16.0, 2.0 ** -10
    got = windq.windq_gated_grad(*(c.packed for c in cs), dh, g, u)
    want, off = backward(cs, dh, g, u, "silu", BF)
    for a, b, o in zip(got, want, off):
        close(a, b, o, BF)


@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** -100])
def test_tokens_at_both_ends_of_the_range(windq, size):
    shape = (64, 256, 64, 0, 400)
    cs = pair(windq, shape, BF)
    x = tokens(400, 256, BF, 1)
    x[::3] *= size
    save = torch.empty(2, 400, 64, dtype=BF, device=DEV)
    windq.windq_gated(*(c.packed for c in cs), x, save=(save[0], save[1]))
    want, off = forward(cs, x, "silu", BF)
    close(save[0], want[0], off[0] + 2.0 ** -133, BF)
    close(save[1], want[1], off[1] + 2.0 ** -133, BF)


@pytest.mark.parametrize("shape", GATED)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_token_that_is_not_finite_is_nobody_elses(windq, shape, bad):
    *shape, dtype = shape
    cs = pair(windq, shape, dtype)
    p = [c.packed for c in cs]
    rows, cols, T = shape[0], shape[1], shape[4]
    x, dh, g, u = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2), tokens(T, rows, dtype, 3), tokens(T, rows, dtype, 4)
    clean = windq.windq_gated(*p, x), *windq.windq_gated_grad(*p, dh, g, u)
    x[2, cols // 2], dh[1, rows // 3], g[3, rows // 2] = bad, bad, bad
    h, dx, dg, du = windq.windq_gated(*p, x), *windq.windq_gated_grad(*p, dh, g, u)
    others = torch.ones(T, dtype=torch.bool, device=DEV)
    others[2] = False
    assert torch.equal(h[others], clean[0][others]) and not finite(h[2]).any()
    others[2], others[1], others[3] = True, False, False
    assert torch.equal(dx[others], clean[1][others]) and not finite(dx[[1, 3]]).any()
    for got, want in ((dg, clean[2]), (du, clean[3])):
        keep = torch.ones_like(got, dtype=torch.bool)
        keep[1, rows // 3] = keep[3, rows // 2] = False
        assert torch.equal(got[keep], want[keep])
    assert not finite(du[1, rows // 3])


def spoil(windq, c, what, bad):
    """The case's packed matrix with one value that is not finite: -> (packed, row, columns it takes away)."""
    scale, offset, W = c.scale.clone(), c.offset.clone(), c.W.clone()
    nc = c.cols // c.G
    kind = {"scale": lambda a: a != 0, "offset": lambda a: 0 < a < 5, "skip": lambda a: a == 0}[what]
    units = [k for k, a in enumerate(c.action.tolist()) if kind(a)]
    if not units:
        pytest.skip("no unit of the kind in this shape")
    k = units[-1]
    row = k // nc * c.R_u + c.R_u - 1
    lo = k % nc * c.G
    if what == "scale":
        scale.view(-1)[k * c.R_u + c.R_u - 1] = bad
    elif what == "offset":
        offset.view(-1)[k * c.R_u + c.R_u - 1] = bad
    else:
        W[row, lo + 3] = bad
    return c.describe(windq, W=W, scale=scale, offset=offset), row, range(lo + 3, lo + 4) if what == "skip" else range(lo, lo + c.G)


@pytest.mark.parametrize("shape", GATED)
@pytest.mark.parametrize("what", ["scale", "offset", "skip"])
@pytest.mark.parametrize("second", [False, True])
def test_a_weight_that_is_not_finite_is_its_rows_and_columns(windq, shape, what, second):
    *shape, dtype = shape
    cs = pair(windq, shape, dtype)
    rows, cols, T = shape[0], shape[1], shape[4]
    x, dh, g, u = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2), tokens(T, rows, dtype, 3), tokens(T, rows, dtype, 4)
    for bad in (float("nan"), float("inf")):
        p = [c.packed for c in cs]
        p[second], row, taken = spoil(windq, cs[second], what, bad)
        h, (dx, _, _) = windq.windq_gated(*p, x), windq.windq_gated_grad(*p, dh, g, u)
        want, off = forward(cs, x, "silu", dtype)
        rest = np.arange(rows) != row
        close(h[:, torch.from_numpy(rest).to(DEV)], want[2][:, rest], off[2][:, rest], dtype)
        # act(-infinity) is NaN, act(G) times an infinity is not finite
        assert not finite(h[:, row]).any()
        back, boff = backward(cs, dh, g, u, "silu", dtype)
        rest = ~np.isin(np.arange(cols), list(taken))
        close(dx[:, torch.from_numpy(rest).to(DEV)], back[0][:, rest], boff[0][:, rest], dtype)
        assert not finite(dx[:, torch.from_numpy(~rest).to(DEV)]).any()


@pytest.mark.parametrize("shape", EIGHT)
@pytest.mark.parametrize("what", ["token", "scale", "offset", "skip"])
def test_8_bit_products_keep_what_is_not_finite_apart(windq, shape, what):
    *shape, w_dtype = shape
    rows, T = shape[0], shape[4]
    cs, t, _, _ = products(windq, shape, w_dtype, pair=True)
    s = [windq.Serving(c.packed) for c in cs]
    clean = windq.windq_project8(s[0], t, F32), windq.windq_gated8(*s, t, dtype=F32)
    keep, lost = torch.ones(T, rows, dtype=torch.bool, device=DEV), torch.zeros(T, rows, dtype=torch.bool, device=DEV)
    if what == "token":
        x = tokens(T, shape[1], BF, 5)
        x[3, 7] = float("inf")
        t = windq.windq_tokens8(x, shape[2])
        lost[3] = True
    else:
        packed, row, _ = spoil(windq, cs[0], what, float("nan"))
        s[0] = windq.Serving(packed)
        lost[:, row] = True
    keep = ~lost
    for got, want in zip((windq.windq_project8(s[0], t, F32), windq.windq_gated8(*s, t, dtype=F32)), clean):
        assert torch.equal(got[keep], want[keep]) and not finite(got[lost]).any()


@pytest.mark.parametrize("shape", GATED)
def test_malformed_entries_count_as_skip(windq, shape):
    *shape, dtype = shape
    cs = pair(windq, shape, dtype)
    rows, cols, T = shape[0], shape[1], shape[4]
    c = cs[0]
    U = c.action.numel()
    action, off, skips = c.action.clone(), c.off.clone(), c.action.clone()
    bad = {U - 1: ("action", 9)}
    if U > 2:
        bad[0], bad[1] = ("off", -16), ("off", int(c.codes.numel()) + 1024)
    for k, (where, value) in bad.items():
        (action if where == "action" else off)[k] = value
        skips[k] = 0
    malformed = c.describe(windq, action=action.to(DEV), code_off=off.to(DEV))
    plain = c.describe(windq, action=skips.to(DEV))
    x, dh, g, u = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2), tokens(T, rows, dtype, 3), tokens(T, rows, dtype, 4)
    for order in (lambda p: (p, cs[1].packed), lambda p: (cs[1].packed, p)):
        assert torch.equal(windq.windq_gated(*order(malformed), x), windq.windq_gated(*order(plain), x))
        for a, b in zip(windq.windq_gated_grad(*order(malformed), dh, g, u), windq.windq_gated_grad(*order(plain), dh, g, u)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T", [5, 60, 700])
def test_images_that_do_not_belong(windq, T):
    """Units of malformed entries, whose weights stay as they are, with room for them and without; a layout that has no room for a unit's fields; an image whose words say anything."""
    rows, cols, G = (8192, 640, 128) if T == 700 else (256, 640, 128)
    c = Case(windq, rows, cols, G, 0, BF, seed=1)
    assert c.action[1] == 6
    t = windq.windq_tokens8(tokens(T, cols, BF, 3), G)
    q = eight(tokens(T, cols, BF, 3), t.codes.shape[1], G, block(G))[3].astype(float)
    sigma = t.scale.double().cpu().numpy()[:, None]
    broken = c.action.clone()
    broken[1] = 9
    malformed = c.describe(windq, action=broken.to(DEV))
    skips = c.action.clone()
    skips[1] = 0
    w = c.w.copy()
    w[:, G:2 * G] = c.W.double().cpu().numpy()[:, G:2 * G]
    mag = magnitudes(c)
    mag[:, G:2 * G] = np.abs(w[:, G:2 * G])
    mag = EPS * sigma * (np.abs(q) @ mag.T)
    close(windq.windq_project8(windq.Serving(malformed, skips), t, F32), sigma * (q @ w.T), mag, F32)
    w[:, G:2 * G] = 0.0                                    # laid out as it was: fewer bytes than the weights need
    close(windq.windq_project8(windq.Serving(malformed, c.action), t, F32), sigma * (q @ w.T), mag, F32)
    # words and all else at random: whatever comes out, it comes out in its place
    s = windq.Serving(c.packed)
    g = torch.Generator(device=DEV).manual_seed(T)
    s.image.copy_(torch.randint(0, 256, s.image.shape, generator=g, device=DEV, dtype=torch.uint8))
    out = torch.full((T + 2, rows + 8), 3.0, dtype=F32, device=DEV)
    windq.windq_project8(s, t, out=out[1:-1, 4:-4])
    assert torch.all(out[0] == 3.0) and torch.all(out[-1] == 3.0) and torch.all(out[:, :4] == 3.0) and torch.all(out[:, -4:] == 3.0)


@pytest.mark.parametrize("shape", [(64, 4160, 8, 0, 330), (72, 256, 64, 8, 321), (24, 128, 64, 4, 350), (40, 512, 128, 40, 1000), (1001, 512, 128, 0, 400), (8, 8, 8, 0, 1), (1, 8, 8, 1, 3),
                                   (1, 64, 64, 0, 500), (8, 64, 64, 8, 321), (16, 1024, 512, 16, 320)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("masked", [False, True])
def test_small_units_many_chunks_and_the_smallest_sizes(windq, shape, dtype, masked):
    cs = pair(windq, shape, dtype, masked=masked)
    rows, cols, T = shape[0], shape[1], shape[4]
    p = [c.packed for c in cs]
    x, dh = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    save = torch.empty(2, T, rows, dtype=dtype, device=DEV)
    h = windq.windq_gated(*p, x, "gelu", save=(save[0], save[1]))
    want, off = forward(cs, x, "gelu", dtype)
    for got, w, o in zip((save[0], save[1], h), want, off):
        close(got, w, o, dtype)
    got = windq.windq_gated_grad(*p, dh, save[0], save[1], "gelu")
    want, off = backward(cs, dh, save[0], save[1], "gelu", dtype)
    for a, b, o in zip(got, want, off):
        close(a, b, o, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_workspace_for_more_tokens_and_what_lay_in_it(windq, dtype):
    shape = (520, 512, 128, 0, 1000)
    cs = pair(windq, shape, dtype)
    p = [c.packed for c in cs]
    x, dh, g, u = tokens(1000, 512, dtype, 1), tokens(1000, 520, dtype, 2), tokens(1000, 520, dtype, 3), tokens(1000, 520, dtype, 4)
    ws, ws_grad = windq.gated_workspace(*p, x), windq.gated_workspace(*p, dh, grad=True)
    for T in (1, 2, 16, 63, 64, 65, 128, 320, 321, 700, 1000):
        alone = windq.windq_gated(*p, x[:T]), *windq.windq_gated_grad(*p, dh[:T], g[:T], u[:T])
        ws.fill_(255), ws_grad.fill_(255)                  # NaN as half, bfloat16 and fp32
        again = windq.windq_gated(*p, x[:T], ws=ws), *windq.windq_gated_grad(*p, dh[:T], g[:T], u[:T], ws=ws_grad)
        assert all(torch.equal(a, b) for a, b in zip(alone, again)), T


def test_no_tokens(windq):
    cs = pair(windq, (64, 128, 64, 0, 1), BF)
    p, s = [c.packed for c in cs], [windq.Serving(c.packed) for c in cs]
    x, none = torch.empty(0, 128, dtype=BF, device=DEV), torch.empty(0, 64, dtype=BF, device=DEV)
    t = windq.windq_tokens8(x, 64)
    assert t.tokens == 0 and windq.windq_project8(s[0], t).shape == (0, 64) and windq.windq_gated8(*s, t).shape == (0, 64)
    assert windq.windq_gated(*p, x).shape == (0, 64)
    assert [a.shape for a in windq.windq_gated_grad(*p, none, none, none)] == [(0, 128), (0, 64), (0, 64)]


@pytest.mark.parametrize("T", [3, 60, 700])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_windows_of_long_rows(windq, T, dtype):
    """Inputs, outputs and W as windows of tensors with rows of millions of values, offsets past 2^31 and 2^32: the bits of the same values in close rows."""
    rows, cols = 1024, 512
    wide = {3: 1 << 31, 60: 1 << 26, 700: 1 << 23}[T]
    cs = pair(windq, (rows, cols, 128, 0, T), dtype)
    p = [c.packed for c in cs]

    def window(t):
        w = torch.empty(t.shape[0], wide, dtype=t.dtype, device=DEV)[:, wide - 2048:][:, 8:8 + t.shape[1]]
        return w.copy_(t)

    x, dh, g, u = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2), tokens(T, rows, dtype, 3), tokens(T, rows, dtype, 4)
    h = windq.windq_gated(*p, x)
    xw, out = window(x), window(torch.zeros_like(h))
    save = window(torch.zeros_like(h)), window(torch.zeros_like(h))
    plain = torch.empty(2, T, rows, dtype=dtype, device=DEV)
    windq.windq_gated(*p, x, save=(plain[0], plain[1]))
    windq.windq_gated(*p, xw, save=save, out=out)
    assert torch.equal(out, h) and torch.equal(save[0], plain[0]) and torch.equal(save[1], plain[1])
    t, tw = windq.windq_tokens8(x, 128), windq.windq_tokens8(xw, 128)
    assert torch.equal(t.codes, tw.codes) and torch.equal(t.scale, tw.scale) and torch.equal(t.sums, tw.sums)
    s = [windq.Serving(q) for q in p]
    assert torch.equal(windq.windq_project8(s[0], t, out=out), windq.windq_project8(s[0], t, dtype))
    assert torch.equal(windq.windq_gated8(*s, t, out=out), windq.windq_gated8(*s, t, dtype=dtype))
    del xw, out
    want = windq.windq_gated_grad(*p, dh, g, u)
    save[0].copy_(g), save[1].copy_(u)
    dhw = window(dh)
    outs = tuple(window(torch.zeros_like(a)) for a in want)
    assert all(torch.equal(a, b) for a, b in zip(windq.windq_gated_grad(*p, dhw, *save, outs=outs), want))
    del dhw, outs, save
    if T != 3:
        W = torch.empty(rows, 1 << 22, dtype=dtype, device=DEV)[:, (1 << 22) - 1024:][:, :cols]
        far = cs[0].describe(windq, W=W.copy_(cs[0].W))
        assert torch.equal(windq.windq_gated(far, p[1], x), h) and torch.equal(windq.windq_gated_grad(far, p[1], dh, g, u)[0], want[0])
        assert torch.equal(windq.windq_project8(windq.Serving(far), t), windq.windq_project8(s[0], t))


def test_an_image_past_32_bits(windq):
    """Fields behind 2^32 bytes: rows there against the same rows laid out alone."""
    rows, cols, G, unit_rows = 131072, 32768, 128, 4096
    W = torch.empty(rows, cols, dtype=BF, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for part in W.split(8192):
        part.copy_(0.02 * torch.randn(part.shape, generator=g, device=DEV))
    nc, n_rb = cols // G, rows // unit_rows
    action = torch.tensor([(1, 1, 0, 2)[k % 4] for k in range(n_rb * nc)], dtype=torch.uint8)
    cg, idx = torch.tensor([0.9]), torch.zeros(n_rb * nc, 4, dtype=torch.uint8, device=DEV)

    def packed(W, action):
        off = windq.windq_plan_layout(action, unit_rows, G).to(DEV)
        a = action.to(DEV)
        codes, scale, offset = windq.windq_apply_plan(W, G, unit_rows, a, idx[: a.numel()], cg, off)
        return windq.Packed(W, G, unit_rows, a, off, codes, scale, offset)

    x = tokens(700, cols, BF, 2)
    t = windq.windq_tokens8(x, G)
    few = windq.windq_tokens8(x[:3], G)
    s = windq.Serving(packed(W, action), action)
    assert s.image.numel() > 1 << 32
    y, y3 = windq.windq_project8(s, t), windq.windq_project8(s, few, F32)
    h3 = windq.windq_gated8(s, s, few, dtype=F32)
    for rb in (0, n_rb // 2 - 1, n_rb // 2, n_rb - 1):
        mine = slice(rb * unit_rows, (rb + 1) * unit_rows)
        one = windq.Serving(packed(W[mine], action[rb * nc:(rb + 1) * nc]))
        # Another kernel's order: each of them is off by 16 x 2^-24 of its terms' magnitudes, 32768 x 0.2 x |x| (0.8 on average), at most; in H 1.13 |U| and |G| times that.
        off = 2 * EPS * 32768 * 0.2 * 0.9
        a, b = y[:, mine].double(), windq.windq_project8(one, t, F32).double()
        assert torch.all((a - b).abs() <= 2.0 ** -8 * a.abs() + off)
        b = windq.windq_project8(one, few, F32).double()
        assert torch.all((y3[:, mine].double() - b).abs() <= off)
        h = windq.windq_gated8(one, one, few, dtype=F32).double()
        assert torch.all((h3[:, mine].double() - h).abs() <= off * 2.2 * b.abs() + off * off)


@pytest.mark.parametrize("shape", GATED)
def test_captured_and_replayed(windq, shape):
    """Both ways in one graph, and a second one of the same workspace: every replay, with eager work between, is the eager result."""
    *shape, dtype = shape
    rows, cols, T = shape[0], shape[1], shape[4]
    cs = pair(windq, shape, dtype)
    p = [c.packed for c in cs]
    x, dh = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
    save = [torch.empty(2, T, rows, dtype=dtype, device=DEV) for _ in range(2)]
    out = [torch.empty(T, rows, dtype=dtype, device=DEV) for _ in range(2)]
    grads = [tuple(torch.empty(T, w, dtype=dtype, device=DEV) for w in (cols, rows, rows)) for _ in range(2)]
    ws, ws_grad = windq.gated_workspace(*p, x), windq.gated_workspace(*p, dh, grad=True)

    def step(k, word):
        windq.windq_gated(*p, x, word, save=(save[k][0], save[k][1]), ws=ws, out=out[k])
        windq.windq_gated_grad(*p, dh, save[k][0], save[k][1], word, ws=ws_grad, outs=grads[k])

    graphs = []
    for k, word in enumerate(("silu", "gelu")):
        step(k, word)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            step(k, word)
    for again in range(4):
        x.copy_(tokens(T, cols, dtype, 10 + again)), dh.copy_(tokens(T, rows, dtype, 20 + again))
        for k, word in enumerate(("silu", "gelu")):
            ws.fill_(255), ws_grad.fill_(255)
            graphs[k].replay()
        torch.cuda.synchronize()
        for k, word in enumerate(("silu", "gelu")):
            s = torch.empty(2, T, rows, dtype=dtype, device=DEV)
            h = windq.windq_gated(*p, x, word, save=(s[0], s[1]))
            want = windq.windq_gated_grad(*p, dh, s[0], s[1], word)
            assert torch.equal(h, out[k]) and torch.equal(s, save[k]) and all(torch.equal(a, b) for a, b in zip(grads[k], want)), (again, word)


@pytest.mark.parametrize("shape", EIGHT)
def test_8_bit_products_captured_and_replayed(windq, shape):
    *shape, w_dtype = shape
    rows, cols, G, _, T = shape
    cs = [Case(windq, rows, cols, G, shape[3], w_dtype, seed=k) for k in range(2)]
    s = [windq.Serving(c.packed) for c in cs]
    x, t = tokens(T, cols, BF, 1), windq.Tokens8.empty(T, cols, G, DEV)
    y, h = (torch.empty(T, rows, dtype=BF, device=DEV) for _ in range(2))

    def step():
        windq.windq_tokens8(x, G, out=t)
        windq.windq_project8(s[0], t, out=y)
        windq.windq_gated8(*s, t, out=h)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for again in range(4):
        x.copy_(tokens(T, cols, BF, 10 + again))
        t.codes.fill_(1), t.scale.fill_(1.0), t.sums.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        new = windq.windq_tokens8(x, G)
        assert torch.equal(y, windq.windq_project8(s[0], new)) and torch.equal(h, windq.windq_gated8(*s, new))


def test_on_a_stream_of_its_own(windq):
    """Calls wait for nothing but their stream, whose earlier work they see."""
    cs = pair(windq, (512, 512, 128, 0, 400), BF)
    p, s = [c.packed for c in cs], [windq.Serving(c.packed) for c in cs]
    x, dh = tokens(400, 512, BF, 1), tokens(400, 512, BF, 2)
    save = torch.empty(2, 400, 512, dtype=BF, device=DEV)

    def run(x, dh):
        h = windq.windq_gated(*p, x, save=(save[0], save[1]))
        t = windq.windq_tokens8(x, 128)
        return h, *windq.windq_gated_grad(*p, dh, save[0], save[1]), windq.windq_project8(s[0], t), windq.windq_gated8(*s, t)

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
