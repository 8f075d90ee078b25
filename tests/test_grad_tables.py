"""Host checks of the tables that the gradient calls pass on: extents and pitches of pairs of tensors, and the pairs that are refused.
The library is replaced by a recorder, so tensors may be the host's."""
import struct

import pytest
import torch

BF16 = torch.bfloat16


@pytest.fixture
def ws(monkeypatch):
    from paper_2011_09208_amd import buildlib
    if buildlib.is_stale():
        buildlib.build()
    from paper_2011_09208_amd import binding

    class Recorder:
        def __init__(self):
            self.calls = []

        def ws_grad_clip_sgd(self, params, ld_params, param_bytes, grads, rows, cols, lds, elem_bytes, n, *rest):
            q = lambda b: struct.unpack("%dq" % n, b[:8 * n])                                      # noqa: E731
            i = lambda b: struct.unpack("%di" % n, b[:4 * n])                                      # noqa: E731
            self.calls.append((q(params), q(ld_params), i(param_bytes), q(grads), q(rows), q(cols), q(lds), i(elem_bytes)))
            return 0

    monkeypatch.setattr(binding, "lib", Recorder())
    monkeypatch.setattr(binding, "_here", lambda t: t.get_device())
    monkeypatch.setattr(binding, "_stream", lambda: None)
    return binding


def _update(ws, params, grads):
    ws.grad_clip_sgd(params, grads, torch.zeros(1, dtype=torch.float64), 1.0, 0.1)


def _pitched(r, c, dtype=torch.float32):
    return torch.zeros((r, c + 3), dtype=dtype)[:, :c]


@pytest.mark.parametrize("beside", ["nothing", "a contiguous pair", "a pair with a pitch"])
@pytest.mark.parametrize("p,g", [((2, 3), (3, 2)), ((512, 128), (128, 512)), ((2, 3, 2), (12,)), ((6,), (2, 3)), ((2, 3, 2), (2, 6)), ((4, 1), (1, 4)),
                                 ((4, 1), (4,)), ((3,), (4,)), ((0, 8), (8, 0)), ((1, 2, 3), (1, 3, 2))])
def test_pairs_of_other_shapes_are_refused(ws, p, g, beside):
    more = {"nothing": [], "a contiguous pair": [(torch.zeros(5, 7), torch.zeros(5, 7))], "a pair with a pitch": [(torch.zeros(5, 7), _pitched(5, 7))]}[beside]
    for first in (True, False):
        pairs = [(torch.zeros(p), torch.zeros(g, dtype=BF16))] + more
        pairs = pairs if first else pairs[::-1]
        params, grads = [list(x) for x in zip(*pairs)]
        for make in (list, ws.grad_table):
            with pytest.raises(AssertionError):
                _update(ws, make(params), make(grads))
    assert not ws.lib.calls


def test_other_numbers_of_tensors_are_refused(ws):
    a, b = torch.zeros(4, 4), _pitched(4, 4)
    for params, grads in (([a, a], [a]), ([a], [a, a]), ([a], []), ([], [a]), ([a, b], [b]), ([b], [a, b])):
        with pytest.raises(AssertionError):
            _update(ws, params, grads)
    assert not ws.lib.calls


def test_contiguous_pairs_are_long_rows(ws):
    shapes = [(3, 4), (7,), (1, 5), (2, 3, 2), (), (0, 4)]
    params, grads = [torch.zeros(s) for s in shapes], [torch.zeros(s, dtype=BF16) for s in shapes]
    n = tuple(t.numel() for t in params)
    kept = ws.grad_table(params), ws.grad_table(grads)
    for call in ((params, grads), kept, kept):
        _update(ws, *call)
    want = (tuple(t.data_ptr() for t in params), n, (4,) * 6, tuple(t.data_ptr() for t in grads), (1,) * 6, n, n, (2,) * 6)
    assert ws.lib.calls == [want] * 3


def test_pairs_with_a_pitch_are_described_by_their_rows(ws):
    a, pa, b, pb = torch.zeros(3, 4), _pitched(3, 4, BF16), _pitched(6, 2), torch.zeros(6, 2)
    c, pc, d, pd = torch.zeros(2, 3, 2, dtype=BF16), torch.zeros(2, 3, 2), torch.zeros(5), torch.zeros(5)
    _update(ws, [pa, pb, pc, pd], [a, b, c, d])
    got = ws.lib.calls[0]
    assert got[1] == (7, 2, 12, 5) and got[2] == (2, 4, 4, 4) and got[4] == (3, 6, 1, 1) and got[5] == (4, 2, 12, 5)
    assert got[6] == (4, 5, 12, 5) and got[7] == (4, 4, 2, 4)
    ws.lib.calls.clear()
    _update(ws, [a, pb, c, d], [a, pb, c, d])                       # and those without one as one long row
    assert ws.lib.calls[0][4] == (1,) * 4 and ws.lib.calls[0][5] == (12, 12, 12, 5)


@pytest.mark.parametrize("p,g,rows,cols", [((1, 5), (5,), 1, 5), ((5,), (1, 1, 5), 1, 5), ((1, 4, 3), (4, 3), 4, 3), ((), (1,), 1, 1)])
def test_leading_dimensions_of_one_are_left_aside(ws, p, g, rows, cols):
    params, grads = [torch.zeros(p)], [torch.zeros(g)]
    _update(ws, params, grads)
    _update(ws, params + [torch.zeros(5, 7)], grads + [_pitched(5, 7)])
    flat, by_rows = ws.lib.calls
    assert flat[4:7] == ((1,), (rows * cols,), (rows * cols,))
    assert by_rows[4:7] == ((rows, 5), (cols, 7), (cols, 10)) and by_rows[1] == (cols, 7)


def test_more_tensors_than_the_table_of_ones(ws):
    params, grads = [torch.zeros(2, 3)] * 5000, [torch.zeros(2, 3, dtype=BF16)] * 5000
    _update(ws, params, grads)
    assert ws.lib.calls[0][4] == (2,) * 5000 and ws.lib.calls[0][1] == (3,) * 5000


def test_orders_that_a_table_does_not_take(ws):
    for t in (torch.zeros(3, 4).t(), torch.zeros(2, 3, 8)[:, :, :4], torch.zeros(8)[::2]):
        with pytest.raises(AssertionError):
            ws.grad_table([t])
