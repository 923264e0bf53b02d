"""windq_adamw against the formula: bit for bit against its fp32 steps made one by one on the CPU, and against 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn
f32 = np.float32
B1, B2, EPS = 0.9, 0.999, 1e-8


def quantize(x, floor):
    """One rounded operation per step: blocks of 256 over their largest magnitude / 448."""
    n = x.size
    blocks = np.pad(x, (0, -n % 256)).reshape(-1, 256)
    scale = (np.abs(blocks).max(1) * f32(1 / 448)).astype(f32)
    ok = scale >= f32(2.0 ** -126)
    with np.errstate(divide="ignore"):
        inv = np.where(ok, f32(1) / scale, f32(0)).astype(f32)
    scale = np.where(ok, scale, f32(0)).astype(f32)
    q = torch.from_numpy((blocks * inv[:, None]).astype(f32)).to(F8).float().numpy()
    if floor:
        q = np.where((q == 0) & (blocks > 0) & (scale[:, None] > 0), f32(2.0 ** -9), q)
    return q.reshape(-1)[:n].astype(f32), scale


def steps32(p, g, m, v, ms, vs, step, lr, wd, gs, bits):
    """The step in fp32, one rounded operation after the other (inputs as fp32 arrays; 8-bit moments as values and scales)."""
    g = (g * f32(gs)).astype(f32)
    if bits == 8:
        m = (m * np.repeat(ms, 256)[:m.size]).astype(f32)
        v = (v * np.repeat(vs, 256)[:v.size]).astype(f32)
        v = (v * v).astype(f32)
    m = m * f32(B1) + g * f32(1 - B1)
    v = v * f32(B2) + (g * g) * f32(1 - B2)
    root = np.sqrt(v)
    p = p * f32(1 - lr * wd) - (m / (root * f32(1 / np.sqrt(1 - B2 ** step)) + f32(EPS))) * f32(lr / (1 - B1 ** step))
    if bits == 8:
        (m, ms), (v, vs) = quantize(m, False), quantize(root, True)
    return p, m, v, ms, vs


def make(n, bits, p_type, g_type, seed):
    g = torch.Generator().manual_seed(seed)
    size = torch.exp(2 * torch.randn(n, generator=g))
    p = (0.02 * torch.randn(n, generator=g)).to(p_type)
    gr = (1e-3 * size * torch.randn(n, generator=g)).to(g_type)
    m = (1e-4 * size * torch.randn(n, generator=g)).numpy()
    r = (1e-3 * size * torch.rand(n, generator=g)).numpy()
    if bits == 32:
        return p, gr, m, r * r, None, None
    (m, ms), (r, rs) = quantize(m, False), quantize(r, True)
    return p, gr, m, r, ms, rs


def to_dev(x, bits):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(F8) if bits == 8 else t).to(DEV)


def run(windq, sets, bits, step, lr, wd, gs, copies):
    ps, gs_, ms, vs, mss, vss = zip(*sets)
    dev = dict(p=[p.to(DEV) for p in ps], g=[g.to(DEV) for g in gs_], m=[to_dev(m, bits) for m in ms], v=[to_dev(v, bits) for v in vs])
    scales = [[torch.from_numpy(s).to(DEV) for s in x] for x in (mss, vss)] if bits == 8 else [None, None]
    cp = [torch.zeros(p.numel(), dtype=torch.bfloat16, device=DEV) for p in ps] if copies else None
    items = windq.AdamwItems(dev["p"], dev["g"], dev["m"], dev["v"], *scales, cp)
    scale = None if gs is None else torch.tensor([gs], device=DEV)
    windq.windq_adamw(items, step, lr, B1, B2, EPS, wd, grad_scale=scale)
    torch.cuda.synchronize()
    return dev, scales, cp


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_type,g_type", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("sizes", [[1], [255, 256, 257], [4095, 4096, 4097, 3, 8192], [1000 + 37 * i for i in range(75)]])
def test_step_is_the_formulas_fp32_steps(windq, bits, p_type, g_type, sizes):
    for step, lr, wd, gs in ((1, 1e-3, 0.0, None), (137, 3e-2, 0.1, 0.5)):
        sets = [make(n, bits, p_type, g_type, 7 * i + step) for i, n in enumerate(sizes)]
        dev, scales, cp = run(windq, sets, bits, step, lr, wd, gs, p_type == torch.float32)
        for i, (p, g, m, v, ms, vs) in enumerate(sets):
            p64 = p.double().numpy()
            wp, wm, wv, wms, wvs = steps32(p.float().numpy(), g.float().numpy(), m, v, ms, vs, step, lr, wd, 1.0 if gs is None else gs, bits)
            assert torch.equal(dev["p"][i].cpu(), torch.from_numpy(wp).to(p_type))
            assert np.array_equal(dev["m"][i].float().cpu().numpy(), wm) and np.array_equal(dev["v"][i].float().cpu().numpy(), wv)
            if bits == 8:
                assert np.array_equal(scales[0][i].cpu().numpy(), wms) and np.array_equal(scales[1][i].cpu().numpy(), wvs)
            if cp is not None:
                assert torch.equal(cp[i].cpu(), torch.from_numpy(wp).to(torch.bfloat16))
            # the same in 64 bits: the update itself to a few roundings
            g64 = g.double().numpy() * (1.0 if gs is None else gs)
            m64 = m.astype(float) * (np.repeat(ms, 256)[:m.size].astype(float) if bits == 8 else 1)
            v64 = (v.astype(float) * np.repeat(vs, 256)[:v.size].astype(float)) ** 2 if bits == 8 else v.astype(float)
            m1, v1 = B1 * m64 + (1 - B1) * g64, B2 * v64 + (1 - B2) * g64 ** 2
            upd = lr / (1 - B1 ** step) * m1 / (np.sqrt(v1) / np.sqrt(1 - B2 ** step) + EPS)
            p1 = p64 * (1 - lr * wd) - upd
            big = lr / (1 - B1 ** step) * (B1 * np.abs(m64) + (1 - B1) * np.abs(g64)) / (np.sqrt(v1) / np.sqrt(1 - B2 ** step) + EPS)
            out = 2.0 ** -8 if p_type == torch.bfloat16 else 0.0
            tol = 2.0 ** -24 * (4 * np.abs(p64) + 16 * big) + out * np.abs(p1) * (1 + 1e-6)
            assert np.all(np.abs(dev["p"][i].double().cpu().numpy() - p1) <= tol)


def test_many_steps_in_8_bits_stay_near_those_in_32(windq):
    """200 steps of a quadratic: both forms of the moments reach its minimum."""
    g = torch.Generator().manual_seed(3)
    goal = torch.randn(1000, generator=g).to(DEV)
    left = []
    for bits in (32, 8):
        p = torch.zeros(1000, device=DEV)
        m, v = (torch.zeros(1000, device=DEV) if bits == 32 else torch.zeros(1000, dtype=torch.uint8, device=DEV) for _ in range(2))
        scales = [[torch.zeros(4, device=DEV)] for _ in range(2)] if bits == 8 else [None, None]
        grad = torch.empty(1000, device=DEV)
        items = windq.AdamwItems([p], [grad], [m], [v], *scales)
        for step in range(1, 201):
            grad.copy_(p - goal)
            windq.windq_adamw(items, step, 0.05)
        left.append(float((p - goal).norm() / goal.norm()))
    assert left[0] < 0.02 and left[1] < 0.05


@pytest.mark.parametrize("bits", [32, 8])
def test_unaligned_tensors_and_guards(windq, bits):
    """Tensors that start anywhere give the aligned ones' bits, and nothing around them is written."""
    n = 1003
    sets = [make(n, bits, torch.float32, torch.bfloat16, 5)]
    dev, scales, _ = run(windq, sets, bits, 9, 1e-2, 0.01, None, False)
    p, g, m, v, ms, vs = sets[0]

    def at(x, k, fill):
        big = torch.full((n + 16,), fill, device=DEV).to(x.dtype) if x.dtype != F8 else torch.full((n + 16,), 64, dtype=torch.uint8, device=DEV).view(F8)
        big[k:k + n].copy_(x)
        return big

    P, Gr, M, V = at(p.to(DEV), 1, 7.0), at(g.to(DEV), 3, 7.0), at(to_dev(m, bits), 2, 7.0), at(to_dev(v, bits), 5, 7.0)
    more = [[torch.from_numpy(s).to(DEV)] for s in (ms, vs)] if bits == 8 else [None, None]
    items = windq.AdamwItems([P[1:1 + n]], [Gr[3:3 + n]], [M[2:2 + n]], [V[5:5 + n]], *more)
    windq.windq_adamw(items, 9, 1e-2, B1, B2, EPS, 0.01)
    assert torch.equal(P[1:1 + n], dev["p"][0])
    assert torch.equal(M[2:2 + n].float(), dev["m"][0].float()) and torch.equal(V[5:5 + n].float(), dev["v"][0].float())
    for big, k in ((P, 1), (M, 2), (V, 5)):
        around = torch.cat([big[:k].float(), big[k + n:].float()])
        assert torch.all(around == around[0])
    if bits == 8:
        assert torch.equal(more[0][0], scales[0][0]) and torch.equal(more[1][0], scales[1][0])


def test_8_bit_moments_at_the_edges(windq):
    """A block of zeros, one whose scale would be below the normal range, roots too small for their block, NaN and infinities."""
    n = 6 * 256
    g = torch.zeros(n)
    g[256:512] = 1e-38
    g[512] = 1.0
    g[513:768] = 1e-9
    g[768 + 5] = float("nan")
    g[768 + 6:1024] = 1.0
    g[1024 + 7] = float("inf")
    g[1024 + 8:1280] = 1.0
    g[1280:] = 0.25
    sets = [(torch.ones(n), g, np.zeros(n, f32), np.zeros(n, f32), np.zeros(6, f32), np.zeros(6, f32))]
    dev, scales, _ = run(windq, sets, 8, 1, 1e-3, 0.0, None, False)
    p, m, r = dev["p"][0].cpu(), dev["m"][0].float().cpu(), dev["v"][0].float().cpu()
    assert torch.all(p[:256] == 1) and torch.all(m[:256] == 0) and torch.all(r[:256] == 0)
    assert scales[0][0][0] == 0 and scales[1][0][0] == 0
    assert scales[0][0][1] == 0 and torch.all(m[256:512] == 0)
    assert r[512] == 448 and torch.all(r[513:768] == 2.0 ** -9)             # held at the smallest, not lost
    assert torch.isnan(p[768 + 5]) and torch.isnan(m[768 + 5]) and torch.all(torch.isfinite(p[768 + 6:1024]))
    assert torch.isnan(m[1024 + 7]) and torch.all(torch.isfinite(p[1024 + 8:1280]))
    assert torch.all(torch.isfinite(p[1280:])) and torch.all(m[1280:] == 448)


def test_nothing_to_do_and_refusals(windq):
    items = windq.AdamwItems([], [], [], [])
    windq.windq_adamw(items, 1, 1e-3)
    e = lambda n, t=torch.float32: torch.ones(n, dtype=t, device=DEV)  # noqa: E731
    empty = windq.AdamwItems([e(0), e(4)], [e(0), e(4)], [e(0), e(4)], [e(0), e(4)])
    windq.windq_adamw(empty, 1, 1e-3)
    items = windq.AdamwItems([e(4)], [e(4)], [e(4)], [e(4)])
    for bad in (dict(step=0), dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(weight_decay=-1.0)):
        with pytest.raises(windq.WindqError) as x:
            windq.windq_adamw(items, **{"step": 1, "lr": 1e-3, **bad})
        assert x.value.status == windq.WINDQ_EINVAL
    for args, status in ((([e(4)], [e(5)], [e(4)], [e(4)]), windq.WINDQ_ESHAPE), (([e(4)], [], [e(4)], [e(4)]), windq.WINDQ_EINVAL),
                         (([e(4)], [e(4)], [e(4, torch.uint8)], [e(4, torch.uint8)]), windq.WINDQ_EDTYPE),
                         (([e(4)], [e(4)], [e(4, torch.uint8)], [e(4, torch.uint8)], [e(2)], [e(1)]), windq.WINDQ_ESHAPE),
                         (([e(4, torch.float16)], [e(4)], [e(4)], [e(4)]), windq.WINDQ_EDTYPE),
                         (([e(8)[::2]], [e(4)], [e(4)], [e(4)]), windq.WINDQ_ESHAPE)):
        with pytest.raises(windq.WindqError) as x:
            windq.AdamwItems(*args)
        assert x.value.status == status
