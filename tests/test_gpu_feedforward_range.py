"""Values far apart in one call of windq_gated or windq_gated_grad: what goes through half precision is multiplied by powers of two first, and what lies below
them may not be lost where it is the result.

Bounds.  Half a step of 2^-10 a weight (2^-11 of it), dG and dU as well on their way back; of sums 16 x 2^-24 of the magnitudes that are added, as in the calls' own
tests.  What a power leaves no digits for counts as 2^-10 of a result at most, before its own rounding (a bfloat16's half step is 2^-9 to 2^-8); a group of codes
that lies 2^24 and more below its row's largest counts as lost, one above it is off by half a step of 2^-24 at 2^-10: 2^-15 of the group's magnitudes."""
import numpy as np
import pytest
import torch

from test_gpu_eight import act, close
from test_gpu_feedforward_routes import SHAPES
from test_gpu_gated import EPS, curve, pair, slope
from test_gpu_project import DEV, Case, tokens

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def memory():
    """What a test took goes back, for the tests behind it."""
    yield
    torch.cuda.empty_cache()


class Scaled:
    """A case whose weights [row, chunk] are multiplied by powers of two, by their scales and offsets and, where they stay as they are, in W: exact, as long as nothing leaves its type."""

    def __init__(self, windq, c, by):
        nc, R_u = c.cols // c.G, c.R_u
        wide = np.repeat(by, c.G, 1)
        self.w, self.mag = c.w * wide, c.mag * np.abs(wide)
        W = c.W * torch.from_numpy(wide).to(c.W.dtype).to(DEV)
        group = torch.from_numpy(by.reshape(c.rows // R_u, R_u, nc).transpose(0, 2, 1).reshape(-1, R_u)).to(torch.float32).to(DEV)
        scale, offset = ((t.view(-1, R_u) * group).view(-1).contiguous() for t in (c.scale, c.offset))
        self.case, self.W, self.scale, self.offset = c, W, scale, offset
        self.packed = c.describe(windq, W=W, scale=scale, offset=offset)


def scaled(windq, c, rows={}, groups={}):
    """rows: {row: factor}; groups: {(row, chunk): factor}"""
    by = np.ones((c.rows, c.cols // c.G))
    for r, f in rows.items():
        by[r] *= f
    for (r, j), f in groups.items():
        by[r, j] *= f
    return Scaled(windq, c, by)


def products(c, x):
    """(product, how far off it may be before its own rounding) in 64 bits."""
    x = x.double().cpu().numpy()
    y = x @ c.w.T
    return y, (EPS + 2.0 ** -15) * (np.abs(x) @ c.mag.T) + 2.0 ** -11 * (np.abs(x) @ np.abs(c.w).T) + 2.0 ** -10 * np.abs(y)


def saved(windq, cs, x):
    save = torch.empty(2, x.shape[0], cs[0].w.shape[0], dtype=BF, device=DEV)
    windq.windq_gated(cs[0].packed, cs[1].packed, x, save=(save[0], save[1]))
    return save


@pytest.mark.parametrize("shape", SHAPES)
def test_rows_far_apart(windq, shape):
    """Neighbouring rows 2^45 above and 2^40 below the others keep their own digits, and the others theirs."""
    cs = [scaled(windq, c, rows={5: 2.0 ** 45, 6: 2.0 ** -40, shape[0] - 1: 2.0 ** 42, 17 + k: 2.0 ** -50}) for k, c in enumerate(pair(windq, shape, BF))]
    x = tokens(shape[4], shape[1], BF, 4)
    for c, got in zip(cs, saved(windq, cs, x)):
        want, off = products(c, x)
        close(got, want, off, BF)


@pytest.mark.parametrize("up", [2.0 ** 45, 2.0 ** 33, 2.0 ** 27, 2.0 ** 15])
@pytest.mark.parametrize("shape", SHAPES)
def test_groups_far_above_the_rest_of_their_row(windq, shape, up):
    """A row whose largest weights meet zeros of a token is the sum of the others."""
    nc = shape[1] // shape[2]
    cs = [scaled(windq, c, groups={(3, 1): up, (k * 5, nc - 1): up, (20, 0): up, (shape[0] - 2, 0): up}) for k, c in enumerate(pair(windq, shape, BF))]
    x = tokens(shape[4], shape[1], BF, 4)
    for k, j in enumerate((1, nc - 1, 0)):
        x[k::4, j * shape[2]:(j + 1) * shape[2]] = 0.0
    for c, got in zip(cs, saved(windq, cs, x)):
        want, off = products(c, x)
        close(got, want, off, BF)


@pytest.mark.parametrize("up", [2.0 ** 110, 2.0 ** 45, 2.0 ** 33, 2.0 ** 26])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_value_far_above_the_rest_of_its_token(windq, shape, up):
    """What meets a weight of 0 leaves the others to be the sum."""
    rows, cols, G, _, T = shape
    cs = [scaled(windq, c, groups={(r, 1): 0.0 for r in (0, 1, 9, 18, 40, rows - 1 - k)}) for k, c in enumerate(pair(windq, shape, BF))]
    x = tokens(T, cols, BF, 4)
    x[3::7, G + 5] *= up
    x[5, G:2 * G] = up
    for c, got in zip(cs, saved(windq, cs, x)):
        want, off = products(c, x)
        close(got, want, off, BF)


@pytest.mark.parametrize("up", [2.0 ** 37, 2.0 ** 30])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[7]])
def test_values_below_half_precisions_normal_numbers_that_lose_nothing(windq, shape, up):
    """Powers of two next to one far above them: multiples of 2^-24 behind the token's power, which the product takes as they are."""
    rows, cols, G, _, T = shape
    cs = [scaled(windq, c, groups={(r, 1): 0.0 for r in range(0, rows, 3)}) for c in pair(windq, shape, BF)]
    x = tokens(T, cols, BF, 4).sign()
    x[:, G + 5] = up
    for c, got in zip(cs, saved(windq, cs, x)):
        want, off = products(c, x)
        close(got, want, off, BF)


@pytest.mark.parametrize("size", [2.0 ** -80, 2.0 ** 60])
def test_both_at_once_and_small_tokens(windq, size):
    """Rows and tokens of their own ranges: weights and values below what fp32 holds next to them."""
    shape = SHAPES[0]
    rows, cols, G, _, T = shape
    nc = cols // G
    cs = [scaled(windq, c, rows={2: 2.0 ** -60}, groups={(2, 1): 2.0 ** 110, (11, 2): 2.0 ** 50, (12, 3): 2.0 ** -60}) for c in pair(windq, shape, BF)]
    x = tokens(T, cols, BF, 4, size)
    x[1::5, G:2 * G] = 0.0
    x[2::5, 2 * G:3 * G] = 0.0
    x[0::5, 3 * G + 1] *= 2.0 ** 60
    for c, got in zip(cs, saved(windq, cs, x)):
        want, off = products(c, x)
        assert np.abs(want).max() < 3e38
        close(got, want, off + 2.0 ** -133, BF)


# kernels (as mangled) that the way back takes, and one that it does not; rows, cols, G, unit_rows, tokens; whether a mask lies over the gate
BACK = [(("gated_turn_kernelILb1E", "dx_gemm_kernelILi4ELb1ELb0E"), "gated_join_kernel", (72, 4096, 128, 0, 2048), False),
        (("gated_turn_kernelILb1E", "dx_gemm_kernelILi2ELb1ELb0E"), "gated_join_kernel", (64, 896, 128, 32, 700), False),
        (("gated_turn_kernelILb1E", "dx_gemm_kernelILi2ELb1ELb0E", "gated_join_kernel"), "ILi4ELb1E", (1096, 672, 96, 0, 70), False),
        (("gated_turn_kernelILb0E", "dx_gemm_kernelILi2ELb1ELb0E", "gated_join_kernel"), "ILi4ELb1E", (301, 560, 80, 43, 200), False),
        (("gated_turn_kernelILb0E", "dx_gemm_kernelILi2ELb1ELb0E", "gated_join_kernel"), "ILi4ELb1E", (264, 512, 128, 0, 1), True)]
WAYS = [(shape, masked) for _, _, shape, masked in BACK]


def gradients(cs, dh, g, u, word):
    """dX and how far off it may be before its own rounding in 64 bits.  Slopes are 0 or 1 and no fp32 function rounds them from |G| = 100 on."""
    dh, g, u = (t.double().cpu().numpy() for t in (dh, g, u))
    far = np.abs(g) >= 100
    near = np.where(far, 0.0, g)
    up, y = np.where(far, (g > 0) * 1.0, slope(word, near)), np.where(far, np.maximum(g, 0.0), act(word, near))
    dg, du = dh * u * up, dh * y
    size = np.where(far, np.abs(up), curve(near)), np.where(far, np.abs(y), np.abs(near) * curve(near))
    each = [(dg, EPS * np.abs(dh * u) * size[0], cs[0]), (du, EPS * np.abs(dh) * size[1], cs[1])]
    want = sum(d @ c.w for d, _, c in each)
    # dG, dU and the weights each half a step of 2^-10, all of it in fp32 sums
    off = sum(o @ np.abs(c.w) * (1 + 2.0 ** -9) + (EPS + 2 * 2.0 ** -11 + 2.0 ** -21) * (np.abs(d) @ np.abs(c.w)) + 2.0 ** -14 * (np.abs(d) @ c.mag) for d, o, c in each)
    return want, off + 2.0 ** -10 * np.abs(want)


def back(windq, cs, dh, g, u, word="silu"):
    want, off = gradients(cs, dh, g, u, word)
    close(windq.windq_gated_grad(cs[0].packed, cs[1].packed, dh, g, u, word)[0], want, off + 2.0 ** -133, BF)


@pytest.mark.parametrize("word", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("shape,masked", WAYS)
def test_a_gate_that_is_shut_takes_nothing_from_its_token(windq, shape, masked, word):
    """dH U and dH G far above everything else, where the slope and the activation are 0."""
    rows, cols, _, _, T = shape
    cs = pair(windq, shape, BF, masked=masked)
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    g[::2, 5], u[::2, 5] = -200.0, 2.0 ** 50
    g[::3, 9] = -2.0 ** 60
    back(windq, cs, dh, g, u, word)


@pytest.mark.parametrize("up", [2.0 ** 100, 2.0 ** 45, 2.0 ** 30])
@pytest.mark.parametrize("shape,masked", WAYS)
def test_a_gradient_far_above_the_rest_of_its_token(windq, shape, masked, up):
    """Columns whose weights meet it with 0 are the sum of the others."""
    rows, cols, G, _, T = shape
    nc = cols // G
    cs = [scaled(windq, c, groups={(5, 1): 0.0, (5, nc - 1): 0.0, (rows - 1, 0): 0.0}) for c in pair(windq, shape, BF, masked=masked)]
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    u[::5, 5] *= up
    dh[1::5, 5] *= up
    dh[2::5, rows - 1] *= up
    back(windq, cs, dh, g, u)


@pytest.mark.parametrize("up", [2.0 ** 100, 2.0 ** 45, 2.0 ** 27])
@pytest.mark.parametrize("shape,masked", WAYS)
def test_groups_far_above_the_rest_of_their_chunk(windq, shape, masked, up):
    """Where a token's gradient is 0 in that row the others are its sum; a token of zeros has none at all."""
    rows, cols, G, _, T = shape
    nc = cols // G
    cs = [scaled(windq, c, groups={(7, 1): up, (rows - 2, nc - 1): up if k == 0 else 1.0}) for k, c in enumerate(pair(windq, shape, BF, masked=masked))]
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    dh[::4, 7] = 0.0
    dh[1::4, rows - 2] = 0.0
    dh[2::4, 7], dh[2::4, rows - 2] = 0.0, 0.0
    dh[3::8] = 0.0
    back(windq, cs, dh, g, u)


@pytest.mark.parametrize("up", [2.0 ** 60, 2.0 ** 27])
@pytest.mark.parametrize("shape,masked", WAYS)
def test_one_weight_far_above_its_chunk(windq, shape, masked, up):
    """A weight that stays as it is; the other columns of its chunk keep theirs."""
    rows, cols, G, _, T = shape
    cs = pair(windq, shape, BF, masked=masked)
    for unit, c in [(c.action.tolist().index(0), c) for c in cs if 0 in c.action.tolist()]:
        row, col = unit // (cols // G) * c.R_u + c.R_u // 2, unit % (cols // G) * G + 3
        c.W, c.w = c.W.clone(), c.w.copy()
        c.W[row, col] = up
        c.w[row, col], c.mag[row, col] = up, up
        c.packed = c.describe(windq)
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    back(windq, cs, dh, g, u, "gelu")


@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** 60])
@pytest.mark.parametrize("shape,masked", [WAYS[0], WAYS[2], WAYS[3]])
def test_gradients_and_weights_of_their_own_ranges(windq, shape, masked, size):
    rows, cols, G, _, T = shape
    nc = cols // G
    cs = [scaled(windq, c, groups={(4, 1): 2.0 ** 50, (11, 2): 2.0 ** -60, (12, nc - 1): 2.0 ** 40, (13, nc - 1): 0.0}) for c in pair(windq, shape, BF, masked=masked)]
    dh, g, u = tokens(T, rows, BF, 6, size), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    dh[::3, 4] = 0.0
    dh[1::3, 13] *= 2.0 ** 50
    dh[2::3, 12] *= 2.0 ** -60
    back(windq, cs, dh, g, u, "gelu_tanh")


@pytest.mark.parametrize("only", range(1, 7))
@pytest.mark.parametrize("shape", [(1, 8, 8, 0, 3), (4, 8, 8, 0, 3), (9, 8, 8, 0, 70), (301, 40, 8, 0, 5), (64, 256, 128, 0, 9)])
def test_code_streams_that_end_with_their_last_code(windq, shape, only):
    """Values formed again read codes eight bytes at a time: within the stream, down to one of a byte."""
    from oracle import windq_oracle as O
    rows, cols, G, _, T = shape
    cs = [Case(windq, rows, cols, G, 0, BF, seed=k, only=only) for k in range(2)]
    cs = [scaled(windq, c, rows={rows // 2: 0.0} if rows > 1 else {}) for c in cs]
    end = int(windq.windq_plan_layout(torch.full((cols // G,), only, dtype=torch.uint8), rows, G)[-2]) + O.bytes_per_group(only, G) * rows
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    if rows > 1:
        u[:, rows // 2] = 2.0 ** 50
    packed = [c.case.describe(windq, W=c.W, scale=c.scale, offset=c.offset, codes=c.case.codes[:end].clone()) for c in cs]
    want, off = gradients(cs, dh, g, u, "silu")
    close(windq.windq_gated_grad(packed[0], packed[1], dh, g, u)[0], want, off + 2.0 ** -133, BF)


@pytest.mark.parametrize("shape,masked", WAYS)
def test_columns_of_nothing(windq, shape, masked):
    """Columns that are 0 in every row, beside others of their octet, where tokens have lost something: 0 as they are, and the others from what is there."""
    rows, cols, G, _, T = shape
    cs = pair(windq, shape, BF, masked=masked)
    for c in cs:
        bits = np.zeros((rows, cols), bool) if c.mask is None else (np.unpackbits(c.mask.cpu().numpy(), axis=1, bitorder="little")[:, :cols] == 1)
        bits[:, 3::16] = True
        c.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little")).to(DEV)
        c.W = c.W.clone()
        c.W[:, 3::16] = 0.0                                # in units that stay as they are
        c.w, c.mag = c.w.copy(), c.mag.copy()
        c.w[:, 3::16] = 0.0
        c.mag[:, 3::16] = 0.0
        c.packed = c.describe(windq)
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    dh[:, 5] = 2.0 ** 40
    want, off = gradients(cs, dh, g, u, "silu")
    dx = windq.windq_gated_grad(cs[0].packed, cs[1].packed, dh, g, u)[0]
    close(dx, want, off + 2.0 ** -133, BF)
    assert torch.all(dx[:, 3::16] == 0.0)


@pytest.mark.parametrize("shape", [WAYS[0][0], WAYS[2][0]])
def test_columns_of_nothing_among_weights_that_stay_as_they_are(windq, shape):
    rows, cols, G, _, T = shape
    cs = [Case(windq, rows, cols, G, 0, BF, seed=k, only=0) for k in range(2)]
    for c in cs:
        c.W = c.W.clone()
        c.W[:, 5::8] = 0.0
        c.w, c.mag = c.W.double().cpu().numpy(), c.W.double().abs().cpu().numpy()
        c.packed = c.describe(windq)
    dh, g, u = tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 2.0), tokens(T, rows, BF, 8, 1.5)
    dh[:, 5] = 2.0 ** 40
    want, off = gradients(cs, dh, g, u, "silu")
    dx = windq.windq_gated_grad(cs[0].packed, cs[1].packed, dh, g, u)[0]
    close(dx, want, off + 2.0 ** -133, BF)
    assert torch.all(dx[:, 5::8] == 0.0)


@pytest.mark.parametrize("shape,masked", WAYS)
def test_what_is_formed_again_repeats_itself(windq, shape, masked):
    """Whatever lay in the workspace, eagerly and from a graph."""
    rows, cols, G, _, T = shape
    cs = [scaled(windq, c, groups={(7, 1): 2.0 ** 45, (5, 1): 0.0}) for c in pair(windq, shape, BF, masked=masked)]
    p = [c.packed for c in cs]
    x, dh, g, u = tokens(T, cols, BF, 4), tokens(T, rows, BF, 6, 1e-3), tokens(T, rows, BF, 7, 8.0), tokens(T, rows, BF, 8, 1.5)
    x[::2, G:2 * G], dh[::2, 7], u[1::4, 5] = 0.0, 0.0, 2.0 ** 50
    ws, ws_grad = windq.gated_workspace(*p, x), windq.gated_workspace(*p, dh, grad=True)
    outs = [torch.empty(T, rows, dtype=BF, device=DEV), torch.empty(T, cols, dtype=BF, device=DEV), *(torch.empty(T, rows, dtype=BF, device=DEV) for _ in range(2))]

    def run():
        windq.windq_gated(*p, x, "gelu", ws=ws, out=outs[0])
        windq.windq_gated_grad(*p, dh, g, u, "gelu", ws=ws_grad, outs=tuple(outs[1:]))

    run()
    want = [t.clone() for t in outs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(4):
        ws.fill_((255, 0, 127, 1)[k]), ws_grad.fill_((255, 0, 127, 1)[k])
        run() if k % 2 else graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
        for t in outs:
            t.fill_(3.0)
