"""windq_project and windq_project_grad against the formulas in 64 bits.

Bounds.  A sum in fp32 of terms whose magnitudes add up to M is held to 16 x 2^-24 M: a term's rounding, the three bfloat16 terms of an fp32
operand and the additions' roundings (which are relative to partial sums and of random sign) together stay well below it.  For
the packed product M counts what the instructions really add, scale |f| |x| and |beta| |x| with the off-centre codes f.  bfloat16
outputs add half a unit in their last place (at most 2^-8 |y|: 8 bits of significand); where an intermediate enters an instruction as two bfloat16 terms, 2^-16
of its products; where weights are rounded to bfloat16 (dX in bfloat16), 2^-8 of theirs, every weight and every way of rounding."""
import numpy as np
import pytest
import torch

from oracle import windq_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 16 * 2.0 ** -24
F0 = np.array([0.0, 0.0, 16.0, 8.0, 4.0, 5.0, 0.0])


class Case:
    """A packed matrix with every treatment in it, its weights in 64 bits, and the magnitudes the product adds."""

    def __init__(self, windq, rows, cols, G, unit_rows, dtype=torch.bfloat16, masked=False, seed=0, only=None):
        g = torch.Generator().manual_seed(seed)
        self.W = (0.02 * torch.randn(rows, cols, generator=g)).to(dtype).to(DEV)
        U, self.R_u = windq.n_units(rows, cols, G, unit_rows)
        self.rows, self.cols, self.G, self.unit_rows, nc = rows, cols, G, unit_rows, cols // G
        self.action = torch.tensor([only if only is not None else (u * 5 + seed) % 7 for u in range(U)], dtype=torch.uint8)
        self.off = windq.windq_plan_layout(self.action, self.R_u, G)
        cg = torch.tensor([0.9])
        idx = torch.zeros(U, 4, dtype=torch.uint8, device=DEV)
        self.mask = None
        if masked:
            bits = torch.rand(rows, cols, generator=g) < 0.05
            bits[: min(rows, 3), :G] = True                                  # rows of a chunk with nothing kept
            self.mask = torch.from_numpy(O.pack_mask(~bits.numpy())).to(DEV)
        self.codes, self.scale, self.offset = windq.windq_apply_plan(self.W, G, unit_rows, self.action.to(DEV), idx, cg, self.off.to(DEV), mask=self.mask) \
            if masked else windq.windq_apply_plan(self.W, G, unit_rows, self.action.to(DEV), idx, cg, self.off.to(DEV))
        self.weights(bits.numpy() if masked else None)
        self.packed = self.describe(windq)

    def describe(self, windq, **other):
        t = dict(W=self.W, action=self.action.to(DEV), code_off=self.off.to(DEV), codes=self.codes, scale=self.scale, offset=self.offset, mask=self.mask)
        t.update(other)
        return windq.Packed(t["W"], self.G, self.unit_rows, t["action"], t["code_off"], t["codes"], t["scale"], t["offset"], t["mask"])

    def weights(self, protected):
        w = self.W.double().cpu().numpy()
        self.w, self.mag = w.copy(), np.abs(w)
        codes, off, act = self.codes.cpu().numpy(), self.off.numpy(), self.action.numpy()
        sc, of = (x.double().cpu().numpy().reshape(-1, self.R_u, 1) for x in (self.scale, self.offset))
        nc = self.cols // self.G
        for u, a in enumerate(act):
            if a == 0:
                continue
            nb = O.bytes_per_group(int(a), self.G)
            data = codes[off[u]:off[u] + nb * self.R_u].reshape(self.R_u, nb)
            if a == 5:
                q = np.stack([data // 3 ** k % 3 for k in range(5)], 2).reshape(self.R_u, -1)[:, :self.G].astype(float) - 1
            else:
                b = {1: 8, 2: 4, 3: 3, 4: 2, 6: 1}[int(a)]
                bits = np.unpackbits(data, axis=1, bitorder="little")[:, :self.G * b].reshape(self.R_u, self.G, b)
                q = (bits * (1 << np.arange(b))).sum(2).astype(float)
                q = 2 * q - 1 if a == 6 else q
            o = of[u] if a < 5 else 0.0
            here = np.s_[u // nc * self.R_u:(u // nc + 1) * self.R_u, u % nc * self.G:(u % nc + 1) * self.G]
            self.w[here] = q * sc[u] + o
            f0 = F0[a]
            self.mag[here] = np.abs(sc[u]) * np.abs(q + (4 if a == 5 else f0)) + np.abs(o - f0 * sc[u])
            if protected is not None:
                self.w[here][protected[here]] = 0.0


def tokens(T, width, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(T, width, generator=g)).to(dtype).to(DEV)


class Side:
    """Adapters of several ranks, one of them 0; what lies past a rank is NaN and must not be read."""

    def __init__(self, windq, n, r, rows, cols, dtype, T, seed=1, order="mixed", plain=False):
        g = torch.Generator().manual_seed(seed)
        self.a = (torch.randn(n, r, cols, generator=g) / cols ** 0.5).to(dtype)
        self.b = (0.05 * torch.randn(n, rows, r, generator=g)).to(dtype)
        ranks = [r if plain or k == 0 else (k * 5) % (r + 1) for k in range(n)]
        for k in range(n):
            self.a[k, ranks[k]:] = float("nan")
            self.b[k, :, ranks[k]:] = float("nan")
        self.ranks, self.alpha = ranks, np.ones(n) if plain else (16.0 / np.maximum(1, ranks)).astype(np.float32).astype(float)
        of = torch.randint(-1, n + 1, (T,), generator=g)                      # -1 and n: none
        self.of = (torch.sort(of)[0] if order == "runs" else of).to(torch.int32)
        self.adapters = windq.Adapters(self.a.to(DEV), self.b.to(DEV), None if plain else torch.tensor(self.alpha, dtype=torch.float32, device=DEV),
                                       None if plain else torch.tensor(ranks, dtype=torch.int32, device=DEV))
        self.n, self.r, self.of_dev = n, r, self.of.to(DEV)

    def project(self, x):
        """h, alpha B h and the magnitudes of both."""
        T = x.shape[0]
        h, hm = np.zeros((T, self.r)), np.zeros((T, self.r))
        y, ym = np.zeros((T, self.b.shape[1])), np.zeros((T, self.b.shape[1]))
        for k in range(self.n):
            at, rk = np.flatnonzero(self.of.numpy() == k), self.ranks[k]
            a, b = self.a[k, :rk].double().numpy(), self.b[k, :, :rk].double().numpy()
            h[at, :rk], hm[at, :rk] = x[at] @ a.T, np.abs(x[at]) @ np.abs(a).T
            y[at], ym[at] = self.alpha[k] * (h[at, :rk] @ b.T), self.alpha[k] * (hm[at, :rk] @ np.abs(b).T)
        return h, hm, y, ym

    def grad(self, x, dy):
        T, C = x.shape
        dx, dxm = np.zeros((T, C)), np.zeros((T, C))
        da, dam = np.zeros((self.n, self.r, C)), np.zeros((self.n, self.r, C))
        db, dbm = np.zeros((self.n, dy.shape[1], self.r)), np.zeros((self.n, dy.shape[1], self.r))
        for k in range(self.n):
            at, rk, al = np.flatnonzero(self.of.numpy() == k), self.ranks[k], self.alpha[k]
            a, b = self.a[k, :rk].double().numpy(), self.b[k, :, :rk].double().numpy()
            d, dm = al * (dy[at] @ b), al * (np.abs(dy[at]) @ np.abs(b))
            dx[at], dxm[at] = d @ a, dm @ np.abs(a)
            da[k, :rk], dam[k, :rk] = d.T @ x[at], dm.T @ np.abs(x[at])
            db[k, :, :rk], dbm[k, :, :rk] = al * dy[at].T @ (x[at] @ a.T), al * np.abs(dy[at]).T @ (np.abs(x[at]) @ np.abs(a).T)
        return dx, dxm, da, dam, db, dbm


def near(got, want, tol):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    worst = np.max(np.abs(got - want) / np.maximum(tol, 1e-300)) if got.size else 0.0
    assert worst <= 1.0, worst


def y_tol(c, x, dtype, want, ym=0.0):
    tol = EPS * (np.abs(x) @ c.mag.T + ym)
    return tol + (2.0 ** -8 * np.abs(want) * 1.001 + 2.0 ** -16 * ym if dtype == torch.bfloat16 else 0.0)


SHAPES = [(512, 512, 128, 0), (200, 384, 64, 0), (192, 256, 128, 64), (100, 960, 96, 0), (60, 80, 8, 20), (33, 240, 40, 11), (48, 1024, 512, 16),
          (264, 512, 256, 0), (7, 64, 32, 1), (1, 128, 128, 0), (1000, 1056, 96, 0), (640, 768, 128, 128), (256, 320, 160, 0)]


@pytest.mark.parametrize("rows,cols,G,unit_rows", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_project_without_adapters(windq, rows, cols, G, unit_rows, dtype):
    for i, T in enumerate((1, 17, 70, 129, 300)):
        c = Case(windq, rows, cols, G, unit_rows, torch.float32 if i % 2 else torch.bfloat16, masked=i == 2, seed=i)
        X = tokens(T, cols, dtype, 50 + i)
        x = X.double().cpu().numpy()
        want = x @ c.w.T
        near(windq.windq_project(c.packed, X), want, y_tol(c, x, dtype, want))


@pytest.mark.parametrize("only", range(7))
def test_project_of_one_treatment(windq, only):
    for w_type in (torch.bfloat16, torch.float32):
        for T, dtype in ((3, torch.float32), (200, torch.bfloat16), (150, torch.float32)):
            c = Case(windq, 320, 512, 128, 0, w_type, seed=only, only=only)
            X = tokens(T, 512, dtype, 9)
            x = X.double().cpu().numpy()
            want = x @ c.w.T
            near(windq.windq_project(c.packed, X), want, y_tol(c, x, dtype, want))


@pytest.mark.parametrize("rows,cols,G,unit_rows", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_project_with_adapters(windq, rows, cols, G, unit_rows, dtype):
    c = Case(windq, rows, cols, G, unit_rows, seed=3)
    for T, n, r, order, plain in ((1, 1, 8, "runs", True), (40, 9, 24, "mixed", False), (65, 3, 64, "mixed", False), (260, 5, 128, "runs", False), (333, 40, 16, "mixed", False)):
        s = Side(windq, n, r, rows, cols, dtype, T, seed=T, order=order, plain=plain)
        X = tokens(T, cols, dtype, T)
        x = X.double().cpu().numpy()
        h, hm, y, ym = s.project(x)
        want = x @ c.w.T + y
        H = torch.full((T, r), float("nan"), device=DEV)
        near(windq.windq_project(c.packed, X, s.adapters, s.of_dev, h=H), want, y_tol(c, x, dtype, want, ym))
        near(H, h, EPS * hm)
        near(windq.windq_project(c.packed, X, s.adapters, s.of_dev), want, y_tol(c, x, dtype, want, ym))


@pytest.mark.parametrize("rows,cols,G,unit_rows", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_grad(windq, rows, cols, G, unit_rows, dtype):
    for i, (T, n, r, order, plain) in enumerate(((1, 1, 8, "runs", True), (40, 9, 24, "mixed", False), (129, 3, 64, "runs", False), (300, 5, 128, "mixed", False))):
        c = Case(windq, rows, cols, G, unit_rows, masked=i == 1, seed=i)
        s = Side(windq, n, r, rows, cols, dtype, T, seed=T, order=order, plain=plain)
        X, dY = tokens(T, cols, dtype, T), tokens(T, rows, dtype, T + 1, 1e-2)
        x, dy = X.double().cpu().numpy(), dY.double().cpu().numpy()
        dx, dxm, da, dam, db, dbm = s.grad(x, dy)
        wm = np.abs(dy) @ c.mag
        want = dy @ c.w + dx
        tol = EPS * (wm + dxm) + (2.0 ** -8 * 1.001 * np.abs(want) + 2.0 ** -8 * (np.abs(dy) @ np.abs(c.w)) + 2.0 ** -16 * dxm if dtype == torch.bfloat16 else 0.0)
        h = torch.empty(T, r, device=DEV)
        windq.windq_project(c.packed, X, s.adapters, s.of_dev, h=h)
        for given in (None, h):
            gx, ga, gb = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev, h=given)
            near(gx, want, tol)
            near(ga, da, EPS * dam)
            near(gb, db, EPS * dbm)
            for k in range(n):                                              # nothing where nothing was trained
                assert torch.all(ga[k, s.ranks[k]:] == 0) and torch.all(gb[k, :, s.ranks[k]:] == 0)
        alone, none_a, none_b = windq.windq_project_grad(c.packed, dY)
        assert none_a is None and none_b is None
        want0 = dy @ c.w
        near(alone, want0, EPS * wm + (2.0 ** -8 * 1.001 * np.abs(want0) + 2.0 ** -8 * (np.abs(dy) @ np.abs(c.w)) if dtype == torch.bfloat16 else 0.0))
        if dtype == torch.bfloat16:                                          # rounded weights cost no more than their size suggests
            assert np.linalg.norm(alone.double().cpu().numpy() - want0) <= 4e-3 * np.linalg.norm(want0)
        side, sa, sb = windq.windq_project_grad(None, dY, X, s.adapters, s.of_dev)
        near(side, dx, EPS * dxm + (2.0 ** -8 * 1.001 * np.abs(dx) + 2.0 ** -16 * dxm if dtype == torch.bfloat16 else 0.0))
        assert torch.equal(sa, ga) or torch.allclose(sa, ga, rtol=0, atol=float(2 * EPS * dam.max()))
        none, ga2, _ = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev, want_dx=False)
        assert none is None and torch.equal(ga2, sa)


def test_gradients_are_the_differences(windq):
    """The loss sum(Y * R) changes along a direction as the gradients say (fp32, central differences of a bilinear function: exact up to rounding)."""
    c = Case(windq, 128, 256, 64, 0, torch.float32, seed=2)
    s = Side(windq, 3, 16, 128, 256, torch.float32, 50, seed=4, plain=True)
    X, R = tokens(50, 256, torch.float32, 1), tokens(50, 128, torch.float32, 2)
    dx, da, db = windq.windq_project_grad(c.packed, R, X, s.adapters, s.of_dev)

    def loss(x, a, b):
        return float((windq.windq_project(c.packed, x, windq.Adapters(a, b), s.of_dev).double() * R.double()).sum())

    A, B = s.a.to(DEV), s.b.to(DEV)
    for k in range(3):
        V = [tokens(50, 256, torch.float32, 20 + k), tokens(3 * 16, 256, torch.float32, 30 + k, 0.06).reshape(3, 16, 256), tokens(3 * 128, 16, torch.float32, 40 + k, 0.05).reshape(3, 128, 16)]
        for i, grad in enumerate((dx, da, db)):
            ends = []
            for e in (0.5, -0.5):
                args = [X, A, B]
                args[i] = args[i] + e * V[i]
                ends.append(loss(*args))
            want = float((grad.double() * V[i].double()).sum())
            size = float((grad.double().abs() * V[i].double().abs()).sum())
            assert abs(ends[0] - ends[1] - want) <= 2e-5 * size + 1e-5 * abs(ends[0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_is_not_finite_stays_in_its_token_and_follows_the_formula(windq, dtype):
    for T in (20, 200):
        c = Case(windq, 256, 512, 128, 0, seed=1)
        X = tokens(T, 512, dtype, 3)
        clean = windq.windq_project(c.packed, X)
        X[2, 40] = float("inf")
        X[3, 300] = float("-inf")
        X[5, 7] = float("nan")
        X[7, 3], X[7, 4] = float("inf"), float("inf")
        X[9] = 1e38
        got = windq.windq_project(c.packed, X).double().cpu().numpy()
        x = X.double().cpu().numpy()
        with np.errstate(all="ignore"):
            for t in (2, 3, 7):
                at = np.flatnonzero(~np.isfinite(x[t]))
                want = (c.w[:, at] * x[t, at]).sum(1)
                assert np.array_equal(np.isnan(want), np.isnan(got[t]))
                assert np.array_equal(want[~np.isnan(want)], got[t][~np.isnan(want)])
            big = x[9] @ c.w.T
            top = float(torch.finfo(dtype).max)
            fine = np.abs(big) < 0.99 * top
            assert np.all(np.isfinite(got[9][fine])) and np.all(np.abs(got[9][fine] - big[fine]) <= 2.0 ** -8 * np.abs(big[fine]) + EPS * (np.abs(x[9]) @ c.mag.T)[fine])
        assert np.all(np.isnan(got[5]))
        rest = [t for t in range(T) if t not in (2, 3, 5, 7, 9)]
        assert np.array_equal(got[rest], clean.double().cpu().numpy()[rest])


def test_malformed_plan_entries_count_as_skip(windq):
    c = Case(windq, 96, 512, 128, 0, seed=1)
    action, off = c.action.clone(), c.off.clone()
    action[0] = 9
    off[1] = off[1] + 8
    off[2] = -16
    off[3] = int(c.codes.numel()) + 16
    packed = c.describe(windq, action=action.to(DEV), code_off=off.to(DEV))
    for T in (5, 150):
        for dtype in (torch.bfloat16, torch.float32):
            X = tokens(T, 512, dtype, 3)
            x = X.double().cpu().numpy()
            want = x @ c.W.double().cpu().numpy().T
            near(windq.windq_project(packed, X), want, y_tol(c, x, dtype, want))
            dY = tokens(T, 96, dtype, 4)
            dy = dY.double().cpu().numpy()
            W = c.W.double().cpu().numpy()
            want = dy @ W
            near(windq.windq_project_grad(packed, dY)[0], want, EPS * (np.abs(dy) @ np.abs(W)) + (2.0 ** -8 * 1.001 * np.abs(want) if dtype == torch.bfloat16 else 0.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_windows_strides_and_guards(windq, dtype):
    """Column windows of wider activations, outputs and gradients give the same bits, and nothing beside them is written."""
    rows, cols = 201, 384
    c = Case(windq, rows, cols, 64, 0, seed=5)
    for T in (30, 190):
        s = Side(windq, 4, 16, rows, cols, dtype, T, seed=2)
        X, dY = tokens(T, cols, dtype, 1), tokens(T, rows, dtype, 2)
        y = windq.windq_project(c.packed, X, s.adapters, s.of_dev)
        grads = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev)
        wide_x = torch.full((T, cols + 24), float("nan"), device=DEV, dtype=dtype)
        wide_x[:, 8:8 + cols] = X
        wide_dy = torch.full((T, rows + 5), float("nan"), device=DEV, dtype=dtype)
        wide_dy[:, 3:3 + rows] = dY
        out = torch.full((T, rows + 6), 7.0, device=DEV, dtype=dtype)
        dx = torch.full((T, cols + 10), 7.0, device=DEV, dtype=dtype)
        xw, dyw, ow, dxw = wide_x[:, 8:8 + cols], wide_dy[:, 3:3 + rows], out[:, 5:5 + rows], dx[:, 1:1 + cols]
        windq.windq_project(c.packed, xw, s.adapters, s.of_dev, out=ow)
        got = windq.windq_project_grad(c.packed, dyw, xw, s.adapters, s.of_dev, outs=(dxw, None, None))
        assert torch.equal(ow, y) and all(torch.equal(a, b) for a, b in zip(got, grads))
        assert torch.all(out[:, :5] == 7) and torch.all(out[:, 5 + rows:] == 7) and torch.all(dx[:, :1] == 7) and torch.all(dx[:, 1 + cols:] == 7)


def test_repeats_streams_and_workspaces(windq):
    """The same bits again, on another stream, and from a workspace full of NaN; a token's result does not depend on its neighbours' values."""
    c = Case(windq, 512, 512, 128, 0, seed=6)
    for T in (12, 400):
        s = Side(windq, 6, 32, 512, 512, torch.bfloat16, T, seed=3)
        X, dY = tokens(T, 512, torch.bfloat16, 1), tokens(T, 512, torch.bfloat16, 2)
        y = windq.windq_project(c.packed, X, s.adapters, s.of_dev)
        g = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            ws = [windq.project_workspace(c.packed, X, s.adapters, grad=k) for k in (False, True)]
            for w in ws:
                w.fill_(255)
            y2 = windq.windq_project(c.packed, X, s.adapters, s.of_dev, ws=ws[0])
            g2 = windq.windq_project_grad(c.packed, dY, X, s.adapters, s.of_dev, ws=ws[1])
        side.synchronize()
        assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(g, g2))


def test_no_tokens(windq):
    c = Case(windq, 64, 128, 64, 0, seed=1)
    s = Side(windq, 2, 8, 64, 128, torch.bfloat16, 4)
    X, dY = tokens(0, 128, torch.bfloat16, 1), tokens(0, 64, torch.bfloat16, 1)
    of = torch.zeros(0, dtype=torch.int32, device=DEV)
    assert windq.windq_project(c.packed, X, s.adapters, of).shape == (0, 64)
    dx, da, db = windq.windq_project_grad(c.packed, dY, X, s.adapters, of)
    assert dx.shape == (0, 128) and torch.all(da == 0) and torch.all(db == 0)


def test_the_step_replays_from_a_hip_graph(windq):
    """Forward, backward and the optimizer's step of an adapter in one graph: every replay is the eager step's."""
    c = Case(windq, 512, 384, 128, 0, seed=6)
    T = 200
    s = Side(windq, 4, 16, 512, 384, torch.bfloat16, T, seed=3, plain=True)
    X, dY = tokens(T, 384, torch.bfloat16, 1), tokens(T, 512, torch.bfloat16, 2)
    ws = [windq.project_workspace(c.packed, X, s.adapters, grad=k) for k in (False, True)]

    def state():
        p = [s.a.float().to(DEV), s.b.float().to(DEV)]
        return dict(p=p, copy=[s.a.to(DEV).clone(), s.b.to(DEV).clone()], g=[torch.zeros_like(t) for t in p], m=[torch.zeros_like(t) for t in p],
                    v=[torch.zeros_like(t) for t in p], y=torch.empty(T, 512, dtype=torch.bfloat16, device=DEV), dx=torch.empty_like(X), h=torch.empty(T, 16, device=DEV))

    def step(t, ad, items):
        windq.windq_project(c.packed, X, ad, s.of_dev, h=t["h"], ws=ws[0], out=t["y"])
        windq.windq_project_grad(c.packed, dY, X, ad, s.of_dev, h=t["h"], ws=ws[1], outs=(t["dx"], t["g"][0], t["g"][1]))
        windq.windq_adamw(items, 3, 1e-3)

    def handles(t):
        return windq.Adapters(*t["copy"]), windq.AdamwItems(t["p"], t["g"], t["m"], t["v"], copies=t["copy"])

    eager, graph = state(), state()
    he, hg = handles(eager), handles(graph)
    warm = state()
    step(warm, *handles(warm))
    torch.cuda.synchronize()
    G = torch.cuda.CUDAGraph()
    with torch.cuda.graph(G):
        step(graph, *hg)
    for _ in range(4):
        step(eager, *he)
        G.replay()
        torch.cuda.synchronize()
        for k in ("y", "dx", "h"):
            assert torch.equal(eager[k], graph[k])
        for k in ("p", "g", "m", "v", "copy"):
            assert all(torch.equal(a, b) for a, b in zip(eager[k], graph[k]))
        junk = torch.randn(1 << 20, device=DEV).sum()                      # eager work of its own between the replays
        assert bool(torch.isfinite(junk))
