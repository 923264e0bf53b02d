"""The adapter calls' Python side without a GPU: what it refuses before the library is called, and the leading dimensions it passes on."""
import pytest
import torch

BF = torch.bfloat16
ROWS, COLS, G = 64, 128, 64


class Library:
    """Takes the calls in the library's place, and keeps their arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def library(windq, monkeypatch):
    L = Library()
    monkeypatch.setattr(windq.binding, "_require_cuda", lambda *ts: None)
    monkeypatch.setattr(windq.binding, "_packed", lambda: L)
    monkeypatch.setattr(windq.binding, "_stream", lambda: 0)
    return L


def packed_matrix(windq):
    U = COLS // G
    return windq.Packed(torch.zeros(ROWS, COLS, dtype=BF), G, 0, torch.zeros(U, dtype=torch.uint8), torch.zeros(U + 1, dtype=torch.int64),
                        torch.zeros(16, dtype=torch.uint8), torch.zeros(U * ROWS), torch.zeros(U * ROWS))


@pytest.mark.parametrize("grad", [False, True])
def test_outputs_whose_rows_overlap_are_refused(windq, library, grad):
    packed, width = packed_matrix(windq), COLS if grad else ROWS
    f = windq.windq_project_grad if grad else windq.windq_project
    x = lambda T: torch.zeros(T, ROWS if grad else COLS, dtype=BF)  # noqa: E731
    out = lambda t: {"outs": (t, None, None)} if grad else {"out": t}  # noqa: E731
    for overlapping in (torch.zeros(width, dtype=BF).expand(5, width), torch.zeros(5 * width, dtype=BF).as_strided((5, width), (width - 8, 1)),
                        torch.zeros(width + 4, dtype=BF).as_strided((5, width), (1, 1))):
        with pytest.raises(windq.WindqError) as e:
            f(packed, x(5), **out(overlapping))
        assert e.value.status == windq.WINDQ_ESHAPE and not library.calls
    at = 7 if grad else 5                                # the leading dimension among the arguments
    for T, stride, ld in ((5, width, width), (5, width + 3, width + 3), (1, 0, width), (1, width + 40, width + 40), (0, width, width)):
        f(packed, x(T), **out(torch.zeros(5 * (width + 40), dtype=BF).as_strided((T, width), (stride, 1))))
        name, args = library.calls.pop()
        assert args[at] == ld, (T, stride)
