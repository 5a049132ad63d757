"""Routing and clipping on the host, without a GPU: the bound on a plan's rows
against the definition, workspace sizes, and the arguments that the library and
the binding refuse before anything reaches the device."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2204_05436_amd import hotline as hl


@pytest.mark.parametrize("capacity", [0, 1, 3, 100])
@pytest.mark.parametrize("align", [1, 2, 7, 16])
def test_rows_bound(capacity, align):
    """No ids need more rows than hl_route_rows says, and some need as many: the worst spread of n assignments over
    the experts, by trying every split of small ones."""
    for n_tokens, k, n_experts in [(0, 1, 3), (1, 1, 1), (1, 2, 4), (3, 2, 2), (5, 1, 3), (4, 2, 3), (7, 1, 1)]:
        n = n_tokens * k
        need = 0

        def rows(counts):
            kept = [min(c, capacity) if capacity else c for c in counts]
            return sum(-(-c // align) * align for c in kept)

        def splits(left, parts):
            if parts == 1:
                yield (left,)
                return
            for c in range(left + 1):
                for rest in splits(left - c, parts - 1):
                    yield (c,) + rest

        for total in range(n + 1):  # (some of them padding)
            need = max([need] + [rows(s) for s in splits(total, n_experts)])
        got = hl.hl_route_rows(n_tokens, k, n_experts, capacity, align)
        assert got >= need
        assert got <= need + n_experts * align  # (the bound is near)


def test_sizes_out_of_range():
    for args in [(-1, 1, 1, 0, 1), (1, 0, 1, 0, 1), (1, 1, 0, 0, 1), (1, 1, 1, -1, 1), (1, 1, 1, 0, 0),
                 (1 << 31, 1, 1, 0, 1), (1 << 30, 2, 1, 0, 1)]:
        assert hl.hl_route_rows(*args) == 0
    assert hl.hl_route_workspace_bytes(1, 1, 1025) == 0
    assert hl.hl_route_workspace_bytes(-1, 1, 8) == 0
    assert hl.hl_route_workspace_bytes(4096, 8, 64) > 0
    assert hl.hl_grad_workspace_bytes() > 16384


def test_null_handle_is_refused():
    L = hl.lib()
    r = hl.RouteStruct(1, 1, 1, 0, 1, 1, 1, 1, 1, None)
    assert L.hl_route_plan(None, C.byref(r), None, None, 0, None) == 1
    assert L.hl_route_gather(None, C.byref(r), 0, 1, None, 1, None, 1, None) == 1
    assert L.hl_route_gather_bwd(None, C.byref(r), 0, 1, None, 1, None, 1, None) == 1
    assert L.hl_route_combine(None, C.byref(r), 0, 1, None, 1, None, None, 1, None) == 1
    assert L.hl_route_combine_bwd(None, C.byref(r), 0, 1, None, 1, None, 1, None, None, 1, None, None) == 1
    assert L.hl_grad_sq(None, None, 0, None, None, 0, None) == 1
    assert L.hl_grad_clip(None, None, 0, None, 1, 1.0, None, None) == 1
    assert L.hl_embbag_bwd_norm(None, 0, 1, 1, 1, None, None, None, 0, None) == 1
    assert L.hl_embbag_bwd_clip(None, None, None, 0, 1, 1, 1, None, 1, 1.0, 0.1, None, 0, None, None) == 1


def _route(**kw):
    a = dict(n_tokens=4, k=2, n_experts=3, counts=torch.zeros(3, dtype=torch.int32),
             offsets=torch.zeros(4, dtype=torch.int32), pos=torch.zeros(8, dtype=torch.int32))
    a.update(kw)
    return hl.Route(**a)


def test_binding_refuses_route_arrays():
    _route()
    i32 = dict(dtype=torch.int32)
    for bad in [dict(counts=torch.zeros(2, **i32)), dict(offsets=torch.zeros(3, **i32)),
                dict(pos=torch.zeros(7, **i32)), dict(pos=torch.zeros(8, dtype=torch.int64)),
                dict(pos=torch.zeros(16, **i32)[::2]), dict(order=torch.zeros(5, dtype=torch.int64)),
                dict(order=torch.zeros(5, **i32), n_rows=9)]:
        with pytest.raises(ValueError):
            _route(**bad)


class _Handle:
    ptr = None


def test_binding_refuses_rows_and_weights():
    r, h = _route(), _Handle()
    x, rows, w = torch.zeros(4, 6), torch.zeros(8, 6), torch.zeros(4, 2)
    for a, b in [(torch.zeros(3, 6), rows), (x, torch.zeros(7, 6)), (x, torch.zeros(8, 5)), (x, rows.double()),
                 (torch.zeros(6, 4).t(), rows), (torch.zeros(24), rows)]:
        with pytest.raises(ValueError):
            hl.hl_route_gather(h, r, a, b)
    with pytest.raises(ValueError):
        hl.hl_route_combine(h, r, rows, w.double(), x)
    with pytest.raises(ValueError):
        hl.hl_route_combine(h, r, rows, torch.zeros(7), x)
    with pytest.raises(ValueError):
        hl.hl_route_combine_bwd(h, r, x, rows, w, torch.zeros(8, 6), torch.zeros(2, 4).t()[:3])
    with pytest.raises(ValueError):
        hl.hl_route_plan(h, r, torch.zeros(4, 2, dtype=torch.int64))
    with pytest.raises(TypeError):
        hl.hl_route_gather(h, r, x.double(), rows.double(), stream=0)


def test_binding_refuses_gradients():
    a, b = torch.zeros(4), torch.zeros(3, dtype=torch.bfloat16)
    assert len(hl.GradList([a, b])) == 2 and len(hl.GradList([])) == 0
    for g, o in [([a], []), ([a], [b]), ([a[::2]], None), ([a], [torch.zeros(8)[::2]])]:
        with pytest.raises(ValueError):
            hl.GradList(g, o)
    with pytest.raises(TypeError):
        hl.GradList([torch.zeros(4, dtype=torch.float64)])
    # the same tensor twice, or an output inside what another entry reads or writes
    x, y = torch.zeros(16), torch.zeros(16)
    for g, o in [([x, x], None), ([x[:8], x[4:12]], None), ([x, x[2:4]], None), ([x[:8], x[8:]], [y[:8], x[:8]]),
                 ([x[:8], x[8:]], [y[:8], y[7:15]]), ([x[:8]], [x[4:12]]), ([x, y[:4]], [y, y[:4]])]:
        with pytest.raises(ValueError):
            hl.GradList(g, o)
    for g, o in [([x[:8], x[8:]], None), ([x[:8], x[8:]], [y[:8], y[8:]]), ([x, x[:0]], None), ([x, x], [y, torch.zeros(16)]),
                 ([x[:8], x[8:]], [x[:8], y[:8]]), ([x[:8], x[8:], y], [x[:8], x[8:], y])]:
        hl.GradList(g, o)
    with pytest.raises(ValueError):
        hl.hl_grad_sq(_Handle(), hl.GradList([a]), torch.zeros(1), torch.zeros(8, dtype=torch.uint8), stream=0)
    with pytest.raises(ValueError):
        hl.hl_grad_clip(_Handle(), hl.GradList([a]), torch.zeros(1), 1.0, stream=0)


def test_structs_match_the_header():
    """The binding's structs against the C ones, laid out by the rules of the C ABI."""
    assert C.sizeof(hl.RouteStruct) == 8 + 4 * 4 + 8 + 4 * 8 and hl.RouteStruct.n_rows.offset == 24
    assert C.sizeof(hl.GradStruct) == 32 and hl.GradStruct.dtype.offset == 24
    assert np.dtype(np.int32).itemsize == C.sizeof(C.c_int32)
