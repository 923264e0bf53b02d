"""windq_project, windq_project_grad and windq_adamw without a GPU: every refusal, which precedes any launch, and what the
workspace function promises.  Addresses are made up; a call whose arguments are all right is told apart by what it refuses last, a
workspace that is too small."""
import ctypes

import pytest

AT = 1 << 20                                     # an address on every alignment


def codes_of(windq):
    return {n: getattr(windq, "WINDQ_" + n) for n in ("OK", "EINVAL", "ESHAPE", "EDTYPE", "EWORKSPACE")}


class Call:
    """The arguments of both products as words that a test changes one at a time."""

    def __init__(self, windq):
        B = windq.binding
        self.lib, self.B, self.s = windq.lib(), B, codes_of(windq)
        bf = windq.WINDQ_BF16
        self.W = B.windq_mat(AT, bf, 0, 256, 512, 512)
        self.X = B.windq_mat(AT, bf, 0, 300, 512, 512)
        self.dY = B.windq_mat(AT, bf, 0, 300, 256, 256)
        self.P = B.windq_packed(ctypes.pointer(self.W), None, AT, AT, AT, 1 << 16, AT, AT, 128, 0, 0)
        self.A = B.windq_adapters(AT, AT, AT, AT, 4, 16, bf, 0)
        self.of, self.h, self.Y, self.ld_y, self.dX, self.ld_dx, self.dA, self.dB, self.ws, self.ws_bytes = AT, AT, AT, 256, AT, 512, AT, AT, AT, 256

    def need(self, grad, adapters=True):
        return self.lib.windq_project_workspace_bytes(int(grad), self.X.dtype, self.X.rows, 256, 512, 128, self.A.n if adapters else 0, self.A.max_rank)

    def project(self, P=True, X=True, A=True):
        return self.lib.windq_project(ctypes.byref(self.P) if P else None, ctypes.byref(self.X) if X else None, ctypes.byref(self.A) if A else None,
                                      self.of, self.Y, self.ld_y, self.h, self.ws, self.ws_bytes, None)

    def grad(self, P=True, dY=True, X=True, A=True):
        return self.lib.windq_project_grad(ctypes.byref(self.P) if P else None, ctypes.byref(self.dY) if dY else None, ctypes.byref(self.X) if X else None,
                                           ctypes.byref(self.A) if A else None, self.of, self.h, self.dX, self.ld_dx, self.dA, self.dB, self.ws,
                                           self.ws_bytes, None)


@pytest.fixture
def call(windq):
    return Call(windq)


def test_arguments_that_are_right_get_as_far_as_the_workspace(windq, call):
    s = call.s
    assert call.need(False) > 256 and call.need(True) > 256
    for few in (0, 256, None):
        for grad in (False, True):
            call.ws_bytes = call.need(grad) - 1 if few is None else few
            assert (call.grad() if grad else call.project()) == s["EWORKSPACE"]
    call.ws_bytes = 256
    assert call.project(A=False) == s["EWORKSPACE"] and call.grad(P=False) == s["EWORKSPACE"]
    call.dA = call.dB = None
    assert call.grad(A=False, X=False) == s["EWORKSPACE"]
    call.ws = None
    assert call.project() == s["EWORKSPACE"]
    call.ws, call.ws_bytes = AT + 64, 1 << 30                     # a workspace is on 256 bytes
    assert call.project() == s["EINVAL"] and call.grad() == s["EINVAL"]


def change(c, path, value):
    *at, name = path.split(".")
    o = c
    for n in at:
        o = getattr(o, n)
    setattr(o, name, value)


COMMON = [("P.action", None, "EINVAL"), ("P.code_off", None, "EINVAL"), ("P.codes", None, "EINVAL"), ("P.scale", None, "EINVAL"), ("P.offset", None, "EINVAL"),
          ("P.codes", AT + 8, "EINVAL"), ("P.code_off", AT + 4, "EINVAL"), ("P.scale", AT + 2, "EINVAL"), ("P.offset", AT + 1, "EINVAL"),
          ("P.chunk_w", 0, "ESHAPE"), ("P.chunk_w", 96, "ESHAPE"), ("P.unit_rows", 100, "ESHAPE"), ("P.unit_rows", -1, "ESHAPE"), ("W.dtype", 7, "EDTYPE"),
          ("W.data", None, "EINVAL"), ("W.ld", 511, "ESHAPE"), ("A.a", None, "EINVAL"), ("A.b", None, "EINVAL"), ("A.a", AT + 8, "EINVAL"), ("A.b", AT + 2, "EINVAL"),
          ("A.alpha", AT + 2, "EINVAL"), ("A.rank", AT + 2, "EINVAL"), ("A.dtype", 5, "EDTYPE"), ("A.dtype", "other", "EDTYPE"), ("A.n", 0, "ESHAPE"),
          ("A.n", -3, "ESHAPE"), ("A.n", (1 << 20) + 1, "ESHAPE"), ("A.max_rank", 0, "ESHAPE"), ("A.max_rank", 12, "ESHAPE"), ("A.max_rank", 136, "ESHAPE"),
          ("of", None, "EINVAL"), ("of", AT + 2, "EINVAL"), ("h", AT + 8, "EINVAL"),
          ("X.data", None, "EINVAL"), ("X.data", AT + 8, "EINVAL"), ("X.ld", 504, "ESHAPE"), ("X.ld", 516, "ESHAPE"), ("X.ld", (1 << 31) + 8, "ESHAPE"),
          ("X.cols", 504, "ESHAPE"), ("X.rows", -1, "ESHAPE"), ("X.dtype", 9, "EDTYPE"), ("X.dtype", "other", "EDTYPE")]


@pytest.mark.parametrize("path,value,why", COMMON + [("ld_y", 255, "ESHAPE"), ("ld_y", (1 << 31) + 1, "ESHAPE"), ("Y", None, "EINVAL"), ("Y", AT + 1, "EINVAL"),
                                                     ("X.rows", 1 << 23, "ESHAPE"), ("X.rows", 1 << 31, "ESHAPE")])
def test_windq_project_refuses(windq, call, path, value, why):
    change(call, path, windq.WINDQ_F32 if value == "other" else value)
    assert call.project() == call.s[why]


@pytest.mark.parametrize("path,value,why", COMMON + [("X.rows", 299, "ESHAPE"), ("dY.rows", -1, "ESHAPE"), ("dY.cols", 255, "ESHAPE"), ("dY.ld", 255, "ESHAPE"),
                                                     ("dY.data", None, "EINVAL"), ("dY.data", AT + 1, "EINVAL"), ("dY.dtype", 3, "EDTYPE"), ("dY.rows", 1 << 22, "ESHAPE"),
                                                     ("dA", None, "EINVAL"), ("dB", None, "EINVAL"), ("dA", AT + 8, "EINVAL"), ("dB", AT + 4, "EINVAL"),
                                                     ("dX", AT + 1, "EINVAL"), ("ld_dx", 511, "ESHAPE"), ("ld_dx", (1 << 31) + 1, "ESHAPE")])
def test_windq_project_grad_refuses(windq, call, path, value, why):
    change(call, path, windq.WINDQ_F32 if value == "other" else value)
    assert call.grad() == call.s[why]


def test_what_may_be_left_out_and_what_may_not(windq, call):
    s = call.s
    assert call.project(P=False) == s["EINVAL"] and call.project(X=False) == s["EINVAL"]
    assert call.grad(dY=False) == s["EINVAL"] and call.grad(X=False) == s["EINVAL"] and call.grad(A=False) == s["EINVAL"]
    assert call.grad(P=False, X=False) == s["EINVAL"]             # nothing says how many columns there are
    call.dX = None
    assert call.grad() == s["EWORKSPACE"]
    call.dA = call.dB = None
    assert call.grad() == s["EINVAL"]                             # nothing is wanted
    call.dX = AT
    assert call.grad(X=False) == s["EWORKSPACE"]                  # dX alone needs no X
    call.W.data, call.h = AT, None
    assert call.grad() == s["EWORKSPACE"] and call.project() == s["EWORKSPACE"]


def test_no_tokens_are_no_work(windq, call):
    call.X.rows = call.dY.rows = 0
    call.X.data = call.dY.data = call.of = call.Y = None
    call.ws = None
    assert call.project() == call.s["OK"]
    assert call.grad() == call.s["EWORKSPACE"]                    # the adapters' gradients are still written, as zeros


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("rows,cols,G,n,rank", [(256, 512, 128, 0, 0), (4096, 4096, 128, 1, 64), (1000, 1056, 96, 5, 24), (512, 11008, 128, 30, 128), (33, 240, 40, 3, 8)])
def test_a_workspace_for_more_tokens_does_for_fewer(windq, grad, rows, cols, G, n, rank):
    f = windq.lib().windq_project_workspace_bytes
    for dtype in (windq.WINDQ_BF16, windq.WINDQ_F32):
        sizes = [f(grad, dtype, T, rows, cols, G, n, rank) for T in list(range(0, 700)) + list(range(701, 9000, 37))]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_workspace_of_sizes_out_of_range(windq):
    f, B = windq.lib().windq_project_workspace_bytes, windq.WINDQ_BF16
    assert f(0, B, 10, 256, 512, 128, 4, 16) > 0
    for bad in ((0, 2, 10, 256, 512, 128, 4, 16), (0, B, -1, 256, 512, 128, 4, 16), (0, B, 10, 0, 512, 128, 4, 16), (0, B, 10, 256, 0, 128, 4, 16),
                (0, B, 10, 256, 512, 0, 4, 16), (0, B, 10, 256, 512, 128, -1, 16), (0, B, 10, 256, 512, 128, 4, 136), (1, B, 1 << 31, 256, 512, 128, 4, 16),
                (1, B, 10, (1 << 31) + 1, 512, 128, 4, 16), (1, B, 10, 256, (1 << 31) + 8, 128, 4, 16)):
        assert f(*bad) == 0


def adamw(windq, n=1, p=None, g=None, bits=32, step=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, scale=None, items=True, **item):
    words = dict(p=AT, g=AT, m=AT, v=AT, m_scale=AT, v_scale=AT, copy=None, n=0)
    words.update(item)
    one = windq.binding.windq_adamw_item(*(words[k] for k in ("p", "g", "m", "v", "m_scale", "v_scale", "copy", "n")))
    F = windq.WINDQ_F32
    return windq.lib().windq_adamw(ctypes.byref(one) if items else None, n, F if p is None else p, F if g is None else g, bits, step, lr, b1, b2, eps, wd, scale, None)


def test_windq_adamw_refuses(windq):
    s, nan, inf = codes_of(windq), float("nan"), float("inf")
    assert adamw(windq) == s["OK"] and adamw(windq, bits=8) == s["OK"] and adamw(windq, n=0, items=False) == s["OK"]        # n = 0 in the item, or no item
    for wrong in (dict(n=-1), dict(items=False), dict(bits=16), dict(step=0), dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0),
                  dict(b2=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=inf), dict(eps=1e-60), dict(wd=-0.1), dict(wd=nan), dict(scale=AT + 2)):
        assert adamw(windq, **wrong) == s["EINVAL"], wrong
    assert adamw(windq, p=7) == s["EDTYPE"] and adamw(windq, g=7) == s["EDTYPE"]


@pytest.mark.parametrize("bits", [32, 8])
def test_windq_adamw_refuses_an_item(windq, bits):
    s, B = codes_of(windq), windq.binding
    def item(**w):
        one = B.windq_adamw_item(*(dict(dict(p=AT, g=AT, m=AT, v=AT, m_scale=AT, v_scale=AT, copy=None, n=100), **w)[k]
                                   for k in ("p", "g", "m", "v", "m_scale", "v_scale", "copy", "n")))
        return windq.lib().windq_adamw(ctypes.byref(one), 1, windq.WINDQ_F32, windq.WINDQ_BF16, bits, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, None, None)
    for k in ("p", "g", "m", "v"):
        assert item(**{k: None}) == s["EINVAL"]
    assert item(n=-1) == s["ESHAPE"] and item(n=1 << 62) == s["ESHAPE"]
    assert item(p=AT + 2) == s["EINVAL"] and item(g=AT + 1) == s["EINVAL"] and item(copy=AT + 1) == s["EINVAL"]
    if bits == 32:
        assert item(m=AT + 2) == s["EINVAL"] and item(v=AT + 1) == s["EINVAL"]
    else:
        assert item(m_scale=None) == s["EINVAL"] and item(v_scale=None) == s["EINVAL"] and item(m_scale=AT + 2) == s["EINVAL"]
