"""windq_tokens8, windq_serving_layout, windq_serving_lay, windq_project8, windq_gated8, windq_gated and windq_gated_grad without a GPU: every refusal, which
precedes any launch, and the host functions' values.  Addresses are made up."""
import ctypes

import numpy as np
import pytest
import torch

from test_adapters_binding import Library, packed_matrix  # noqa: F401
from test_adapters_host import AT, change, codes_of

ref = ctypes.byref


class Call:
    """The arguments of all calls as words that a test changes one at a time."""

    def __init__(self, windq):
        B = windq.binding
        self.lib, self.B, self.s, bf = windq.lib(), B, codes_of(windq), windq.WINDQ_BF16
        self.W = B.windq_mat(AT, bf, 0, 256, 512, 512)
        self.V = B.windq_mat(AT, bf, 0, 256, 512, 512)
        self.X = B.windq_mat(AT, bf, 0, 300, 512, 512)
        self.dH = B.windq_mat(AT, bf, 0, 300, 256, 256)
        self.P = B.windq_packed(ctypes.pointer(self.W), None, AT, AT, AT, 1 << 16, AT, AT, 128, 0, 0)
        self.R = B.windq_packed(ctypes.pointer(self.V), None, AT, AT, AT, 1 << 16, AT, AT, 128, 0, 0)
        self.S = B.windq_serving(AT, 1 << 20, 256, 512, 0, 128, bf)
        self.Z = B.windq_serving(AT, 1 << 20, 256, 512, 0, 128, bf)
        self.T = B.windq_tokens(AT, AT, AT, 0, 512, 128, 0)
        self.codes = self.scale = self.sums = self.off = self.image = self.Y = self.G = self.U = self.dX = self.dG = self.dU = self.ws = AT
        self.image_bytes, self.ws_bytes, self.dtype, self.act, self.ld, self.ld_save, self.ld_dx, self.ld_d, self.chunk = 1 << 20, 256, bf, 0, 256, 256, 512, 256, 128

    def tokens8(self):
        return self.lib.windq_tokens8(ref(self.X), self.chunk, self.codes, self.scale, self.sums, None)

    def lay(self):
        return self.lib.windq_serving_lay(ref(self.P), self.off, self.image, self.image_bytes, None)

    def project8(self, P=True, X=True):
        return self.lib.windq_project8(ref(self.S) if P else None, ref(self.T) if X else None, self.Y, self.dtype, self.ld, None)

    def gated8(self, up=True):
        return self.lib.windq_gated8(ref(self.S), ref(self.Z) if up else None, ref(self.T), self.act, self.Y, self.dtype, self.ld, None)

    def gated(self, up=True):
        return self.lib.windq_gated(ref(self.P), ref(self.R) if up else None, ref(self.X), self.act, self.Y, self.ld, self.G, self.U, self.ld_save, self.ws, self.ws_bytes, None)

    def grad(self):
        return self.lib.windq_gated_grad(ref(self.P), ref(self.R), ref(self.dH), self.G, self.U, self.ld_save, self.act, self.dX, self.ld_dx, self.dG, self.dU, self.ld_d, self.ws,
                                         self.ws_bytes, None)


@pytest.fixture
def call(windq):
    return Call(windq)


def test_arguments_that_are_right(windq, call):
    s = call.s
    assert call.project8() == s["OK"] and call.gated8() == s["OK"]                      # no tokens
    assert call.gated() == s["EWORKSPACE"] and call.grad() == s["EWORKSPACE"]
    call.G = call.U = None
    assert call.gated() == s["EWORKSPACE"]
    need = lambda grad: call.lib.windq_gated_workspace_bytes(grad, windq.WINDQ_BF16, 300, 256, 512, 128)  # noqa: E731
    call.G = call.U = AT
    for grad, f in ((0, call.gated), (1, call.grad)):
        call.ws_bytes = need(grad) - 1
        assert f() == s["EWORKSPACE"]
        call.ws, call.ws_bytes = AT + 64, 1 << 30
        assert f() == s["EINVAL"]
        call.ws = None
        assert f() == s["EWORKSPACE"]
        call.ws = AT
    call.X.rows = call.dH.rows = 0
    call.X.data = call.dH.data = call.Y = call.codes = None
    assert call.gated() == s["OK"] and call.grad() == s["OK"] and call.tokens8() == s["OK"]


@pytest.mark.parametrize("path,value,why", [("X.dtype", 7, "EDTYPE"), ("X.data", None, "EINVAL"), ("X.data", AT + 8, "EINVAL"), ("X.ld", 511, "ESHAPE"), ("X.ld", 516, "ESHAPE"),
                                            ("X.rows", -1, "ESHAPE"), ("chunk", 0, "ESHAPE"), ("chunk", 96, "ESHAPE"), ("chunk", 12, "ESHAPE"), ("chunk", 1024, "ESHAPE"),
                                            ("X.cols", 500, "ESHAPE"), ("codes", None, "EINVAL"), ("scale", None, "EINVAL"), ("sums", None, "EINVAL"), ("codes", AT + 8, "EINVAL"),
                                            ("scale", AT + 2, "EINVAL"), ("sums", AT + 4, "EINVAL")])
def test_tokens8_refuses(windq, call, path, value, why):
    change(call, path, value)
    assert call.tokens8() == call.s[why]


PACKED = [("P.action", None, "EINVAL"), ("P.code_off", AT + 4, "EINVAL"), ("P.codes", AT + 8, "EINVAL"), ("P.codes", None, "EINVAL"), ("P.scale", None, "EINVAL"),
          ("P.offset", AT + 1, "EINVAL"), ("P.chunk_w", 96, "ESHAPE"), ("P.unit_rows", 100, "ESHAPE"), ("W.dtype", 7, "EDTYPE"), ("W.data", None, "EINVAL"), ("W.ld", 511, "ESHAPE")]


@pytest.mark.parametrize("path,value,why", PACKED + [("P.mask", AT, "EINVAL"), ("off", None, "EINVAL"), ("off", AT + 4, "EINVAL"), ("image", None, "EINVAL"), ("image", AT + 128, "EINVAL"),
                                                     ("image_bytes", 4096, "EWORKSPACE"), ("image_bytes", (1 << 37) + 256, "ESHAPE")])
def test_serving_lay_refuses(windq, call, path, value, why):
    change(call, path, value)
    assert call.lay() == call.s[why]


PRODUCT = [("S.image", None, "EINVAL"), ("S.image", AT + 64, "EINVAL"), ("S.image_bytes", 1000, "EINVAL"), ("S.image_bytes", (1 << 37) + 1, "ESHAPE"), ("S.rows", 0, "ESHAPE"),
           ("S.cols", 0, "ESHAPE"), ("S.cols", 520, "ESHAPE"), ("S.unit_rows", 100, "ESHAPE"), ("S.unit_rows", -1, "ESHAPE"), ("S.chunk_w", 96, "ESHAPE"), ("S.chunk_w", 4, "ESHAPE"),
           ("S.dtype", 9, "EDTYPE"), ("T.cols", 256, "ESHAPE"), ("T.chunk_w", 64, "ESHAPE"), ("T.tokens", -1, "ESHAPE"), ("T.tokens", 1 << 31, "ESHAPE"), ("dtype", 2, "EDTYPE"),
           ("ld", 255, "ESHAPE"), ("ld", (1 << 31) + 1, "ESHAPE")]
WITH_TOKENS = [("T.codes", None, "EINVAL"), ("T.codes", AT + 8, "EINVAL"), ("T.scale", None, "EINVAL"), ("T.scale", AT + 1, "EINVAL"), ("T.sums", None, "EINVAL"), ("T.sums", AT + 8, "EINVAL"),
               ("Y", None, "EINVAL"), ("Y", AT + 1, "EINVAL")]


@pytest.mark.parametrize("path,value,why", PRODUCT + WITH_TOKENS)
def test_products_of_8_bit_tokens_refuse(windq, call, path, value, why):
    if (path, value, why) in WITH_TOKENS:
        call.T.tokens = 5
    change(call, path, value)
    assert call.project8() == call.s[why] and call.gated8() == call.s[why]


def test_pairs_that_do_not_match_are_refused(windq, call):
    s = call.s
    assert call.project8(P=False) == s["EINVAL"] and call.project8(X=False) == s["EINVAL"] and call.gated8(up=False) == s["EINVAL"] and call.gated(up=False) == s["EINVAL"]
    for path, value, why in (("Z.rows", 512, "ESHAPE"), ("Z.unit_rows", 64, "ESHAPE"), ("Z.cols", 1024, "ESHAPE"), ("Z.chunk_w", 64, "ESHAPE"), ("Z.dtype", windq.WINDQ_F32, "EDTYPE"),
                             ("Z.image", None, "EINVAL"), ("act", 3, "EINVAL"), ("act", -1, "EINVAL")):
        c = Call(windq)
        change(c, path, value)
        assert c.gated8() == s[why], path
    for path, value, why in (("V.rows", 512, "ESHAPE"), ("V.cols", 256, "ESHAPE"), ("R.chunk_w", 64, "ESHAPE"), ("R.unit_rows", 64, "ESHAPE"), ("V.dtype", windq.WINDQ_F32, "EDTYPE"),
                             ("V.data", None, "EINVAL"), ("act", 3, "EINVAL"), ("act", -1, "EINVAL")):
        c = Call(windq)
        change(c, path, value)
        assert c.gated() == s[why] and c.grad() == s[why], path


@pytest.mark.parametrize("path,value,why", PACKED + [("X.dtype", 7, "EDTYPE"), ("X.data", AT + 8, "EINVAL"), ("X.cols", 504, "ESHAPE"), ("X.ld", 516, "ESHAPE"), ("Y", None, "EINVAL"), ("Y", AT + 1, "EINVAL"),
                                                     ("G", None, "EINVAL"), ("U", None, "EINVAL"), ("G", AT + 1, "EINVAL"), ("U", AT + 1, "EINVAL"), ("ld", 255, "ESHAPE"),
                                                     ("ld_save", 255, "ESHAPE"), ("ld_save", (1 << 31) + 1, "ESHAPE"), ("X.rows", 1 << 23, "ESHAPE")])
def test_gated_refuses(windq, call, path, value, why):
    change(call, path, value)
    assert call.gated() == call.s[why]


@pytest.mark.parametrize("path,value,why", PACKED + [("dH.dtype", 7, "EDTYPE"), ("dH.data", None, "EINVAL"), ("dH.data", AT + 1, "EINVAL"), ("dH.cols", 255, "ESHAPE"), ("dH.ld", 255, "ESHAPE"),
                                                     ("dH.rows", 1 << 22, "ESHAPE"), ("G", None, "EINVAL"), ("U", AT + 1, "EINVAL"), ("ld_save", 255, "ESHAPE"), ("ld_dx", 511, "ESHAPE"),
                                                     ("ld_dx", (1 << 31) + 1, "ESHAPE"), ("ld_d", 255, "ESHAPE"), ("dX", AT + 1, "EINVAL"), ("dG", None, "EINVAL"), ("dU", None, "EINVAL"),
                                                     ("dG", AT + 1, "EINVAL")])
def test_gated_grad_refuses(windq, call, path, value, why):
    change(call, path, value)
    assert call.grad() == call.s[why]


def test_gated_grad_needs_something_to_do(windq, call):
    call.dX = call.dG = call.dU = None
    assert call.grad() == call.s["EINVAL"]
    call.dX = AT
    assert call.grad() == call.s["EWORKSPACE"]


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("rows,cols,G", [(256, 512, 128), (4096, 4096, 128), (1000, 1056, 96), (33, 240, 40)])
def test_a_workspace_for_more_tokens_does_for_fewer(windq, grad, rows, cols, G):
    f = windq.lib().windq_gated_workspace_bytes
    for dtype in (windq.WINDQ_BF16, windq.WINDQ_F32):
        sizes = [f(grad, dtype, T, rows, cols, G) for T in list(range(0, 700)) + list(range(701, 9000, 37))]
        assert sizes == sorted(sizes) and sizes[0] > 0
    for bad in ((grad, 2, 10, 256, 512, 128), (grad, 1, -1, 256, 512, 128), (grad, 1, 10, 0, 512, 128), (grad, 1, 10, 256, 0, 128), (grad, 1, 10, 256, 512, 0),
                (grad, 1, 10, 1 << 31, 512, 128)):
        assert f(*bad) == 0


def cut(G):
    steps = -(-G // 32)
    parts = -(-steps // 4)
    return -(-steps // parts), parts


@pytest.mark.parametrize("G", list(range(8, 513, 8)))
def test_widths_of_8_bit_tokens(windq, G):
    S, parts = cut(G)
    assert S <= 4 and 32 * S * parts >= G
    for chunks in (1, 3, 8):
        blocks = parts * chunks
        assert windq.lib().windq_tokens8_width(chunks * G, G) == 32 * S * blocks
        assert windq.lib().windq_tokens8_sums(chunks * G, G) == (blocks + 3) // 4 * 4
    for cols, g in ((G + 1, G), (0, G), (-G, G), (G, G + 1), (G, 0), (1024, 1024)):
        if cols % max(1, g) or cols <= 0 or not 8 <= g <= 512:
            assert windq.lib().windq_tokens8_width(cols, g) == 0 and windq.lib().windq_tokens8_sums(cols, g) == 0


@pytest.mark.parametrize("rows,cols,G,unit_rows", [(256, 512, 128, 0), (200, 480, 96, 40), (7, 64, 32, 1), (72, 80, 8, 0), (96, 1024, 512, 32)])
@pytest.mark.parametrize("f32", [0, 1])
def test_serving_layout(windq, rows, cols, G, unit_rows, f32):
    R_u = unit_rows or rows
    U = rows // R_u * (cols // G)
    action = np.array([(u * 5 + 3) % 7 for u in range(U)], np.uint8)
    off = np.zeros(U + 1, np.int64)
    dtype = windq.WINDQ_F32 if f32 else windq.WINDQ_BF16
    f = lambda a=action, **k: windq.lib().windq_serving_layout(a.ctypes.data, *(dict(rows=rows, cols=cols, G=G, unit_rows=unit_rows, dtype=dtype) | k).values(), off.ctypes.data)  # noqa: E731
    assert f() == windq.WINDQ_OK
    S, parts = cut(G)
    blocks = -(-R_u // 32)
    kbs = rows // R_u * blocks * (cols // G) * parts
    at = -(-kbs * 4 // 256) * 256 + kbs * 256
    size = {0: (6144 if f32 else 2048) * S, 1: 1024 * S, 2: 512 * S, 3: 512 * S, 4: 256 * S, 5: 256 * S, 6: 256 * -(-S // 2)}
    for u in range(U):
        assert off[u] == at
        at += size[int(action[u])] * blocks * parts
    assert off[U] == at + 256
    s = codes_of(windq)
    action[-1] = 7
    assert f() == s["EINVAL"]
    action[-1] = 0
    assert f(rows=0) == s["ESHAPE"] and f(cols=cols + 8 * G + 1) == s["ESHAPE"] and f(G=12) == s["ESHAPE"] and f(unit_rows=rows + 1) == s["ESHAPE"] and f(dtype=5) == s["EDTYPE"]
    assert windq.lib().windq_serving_layout(None, rows, cols, G, unit_rows, dtype, off.ctypes.data) == s["EINVAL"]


@pytest.fixture
def library(windq, monkeypatch):
    L = Library()
    monkeypatch.setattr(windq.binding, "_require_cuda", lambda *ts: None)
    monkeypatch.setattr(windq.binding, "_packed", lambda: L)
    monkeypatch.setattr(windq.binding, "_stream", lambda: 0)
    return L


def test_the_binding_refuses_before_the_library_is_called(windq, library):
    BF, F32 = torch.bfloat16, torch.float32
    p, q = packed_matrix(windq), packed_matrix(windq)                # 64 x 128, chunks of 64
    x = torch.zeros(5, 128, dtype=BF)
    h = lambda dtype=BF, T=5, w=64: torch.zeros(T, w, dtype=dtype)  # noqa: E731
    S, D, V = windq.WINDQ_ESHAPE, windq.WINDQ_EDTYPE, windq.WINDQ_EINVAL

    def refused(status, f, *a, **k):
        with pytest.raises(windq.WindqError) as e:
            f(*a, **k)
        assert e.value.status == status and not library.calls

    refused(V, windq.windq_gated, p, q, x, "relu")
    refused(D, windq.windq_gated, p, q, x, out=h(F32))
    refused(S, windq.windq_gated, p, q, x, out=h(w=65))
    refused(S, windq.windq_gated, p, q, x, out=torch.zeros(64, dtype=BF).expand(5, 64))
    refused(D, windq.windq_gated, p, q, x, save=(h(F32), h(F32)))
    refused(S, windq.windq_gated, p, q, x, save=(h(), h(T=4)))
    refused(S, windq.windq_gated, p, q, x, save=(h(), h(w=80)[:, :64]))                       # strides that differ
    refused(S, windq.windq_gated_grad, p, q, h(w=60), h(), h())
    refused(D, windq.windq_gated_grad, p, q, h(), h(F32), h(F32))
    refused(S, windq.windq_gated_grad, p, q, h(), h(), h(w=80)[:, :64])
    refused(S, windq.windq_gated_grad, p, q, h(), h(), h(), outs=(h(), None, None))
    refused(D, windq.windq_gated_grad, p, q, h(), h(), h(), outs=(None, h(F32), h(F32)))
    refused(V, windq.windq_gated_grad, p, q, h(), h(), h(), "relu")
    refused(S, windq.Tokens8, torch.zeros(5, 120, dtype=torch.int8), torch.zeros(5), torch.zeros(5, 4, dtype=torch.int32), 128, 64)
    refused(D, windq.Tokens8, torch.zeros(5, 128, dtype=torch.uint8), torch.zeros(5), torch.zeros(5, 4, dtype=torch.int32), 128, 64)
    refused(S, windq.Tokens8, torch.zeros(5, 128, dtype=torch.int8), torch.zeros(5), torch.zeros(5, 2, dtype=torch.int32), 128, 64)
    refused(S, windq.Tokens8.empty, 5, 100, 64, "cpu")
    refused(D, windq.Serving, p, torch.zeros(2, dtype=torch.int32))
    refused(S, windq.Serving, p, torch.zeros(1, dtype=torch.uint8))
    refused(V, windq.Serving, p, torch.full((2,), 9, dtype=torch.uint8))
    t = windq.Tokens8.empty(5, 128, 64, "cpu")
    refused(S, windq.windq_tokens8, torch.zeros(4, 128), 64, out=t)
    served = windq.Serving(p)
    library.calls.clear()
    refused(S, windq.windq_project8, served, t, out=h(T=4))
    refused(D, windq.windq_project8, served, t, out=h(torch.float16))
    refused(S, windq.windq_gated8, served, served, t, out=torch.zeros(64, dtype=BF).expand(5, 64))
    refused(V, windq.windq_gated8, served, served, t, "tanh")
    windq.windq_gated_grad(p, q, h(), h(), h(), want_dx=False)         # without dX no workspace either
    name, args = library.calls.pop()
    assert name == "windq_gated_grad" and args[7] is None and args[12] is None
