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
from test_gpu_project import DEV, tokens

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
