"""The clipped table update against the plain one where runs of equal rows span many tiles and their sums cancel to
rounding errors, so that another order of the additions shows: bit for bit where both calls take as many elements per
lane, within the bound of an fp32 sum where they do not.  And which calls may come between the norm and the update."""
import math

import numpy as np
import pytest
import torch

from paper_2204_05436_amd import hotline as hl
from test_clip_gpu import Tables, U

pytestmark = pytest.mark.gpu


def cancelling(t):
    """Every row's gradients add up to nearly nothing: dY of its second half of lookups is that of its first, negated."""
    d = t.dY
    for r in np.unique(t.row):
        at = t.bag[t.row == r]
        half = at.size // 2
        if half:
            d[torch.from_numpy(at[half:2 * half].copy()).cuda()] = -d[torch.from_numpy(at[:half].copy()).cuda()]


# (dt, dim, hot rows of 9): bf16 rows of 40 and 520 elements start at odd multiples of 16 bytes after an odd number of rows
@pytest.mark.parametrize("dt,dim,n_hot,same", [("bf16", 40, 3, False), ("bf16", 520, 3, False), ("bf16", 40, 4, True),
                                               ("bf16", 520, 4, True), ("bf16", 64, 3, True), ("bf16", 36, 4, True),
                                               ("f32", 40, 3, True), ("f32", 6, 4, True)])
def test_cancelling_runs(dt, dim, n_hot, same):
    t = Tables(1, 9, dim, dt, 3000, 0.0, seed=dim + n_hot, hot=(n_hot + 0.5) / 9, alpha=1.3)
    try:
        assert t.n_hot == n_hot
        staging = t.w[n_hot:]
        es = staging.element_size()
        assert same == (staging.data_ptr() % (32 if dt == "bf16" and dim % 8 == 0 else min(16, es * (dim & -dim))) == 0)
        cancelling(t)
        t.w.zero_()
        G, A, n = t.sums()
        assert int((n > 200).sum()) >= 3  # (runs of several tiles of at most 192 lookups)
        t.plan()
        t.norm_()
        off = n[:, None] * U * A  # an fp32 sum of n terms is off by (n - 1) U of their sizes at most
        assert abs(float(t.sq) - float(G.square().sum())) <= float((2 * G.abs() * off + off * off).sum())
        a, b = t.w.clone(), t.w.clone()
        t.clip(a, math.inf, 1.0)
        t.apply(b, 1.0)
        f = torch.finfo(t.w.dtype)
        for w in (a, b):  # the rows were zero: the sum, rounded to the type
            assert bool(((w.double() + G).abs() <= off + f.eps / 2 * (G.abs() + off)).all())
        assert bool((a != 0).any())
        if same:
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
            m = float(np.float32(math.sqrt(float(t.sq)) / 7))
            c = np.float32(m / math.sqrt(float(t.sq)))
            a, b = t.w.clone(), t.w.clone()
            t.clip(a, m, 0.25)
            t.apply(b, float(np.float32(0.25) * c))
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()


def test_calls_in_between():
    """The plain update and the grouping keep the norm's sums; calls that write the workspace's buffers lose them."""
    t = Tables(3, 200, 16, "f32", 300, 2.0, seed=4)
    try:
        i32 = dict(dtype=torch.int32, device="cuda")
        w, other = t.w.clone(), t.w.clone()
        keys, bags = torch.zeros(t.L, **i32), torch.zeros(t.L, **i32)
        t.plan()
        t.norm_()
        t.clip(w, 1.0, 0.5)
        keep = lambda: t.apply(other, 0.1), lambda: hl.hl_embbag_bwd_grouping(t.h, *t.shape(), t.ws, keys, bags)
        for f in keep:
            f()
            again = t.w.clone()
            t.clip(again, 1.0, 0.5)
            assert torch.equal(again, w)
        assert not torch.equal(w, t.w)
        k, E = 8, 16
        route = hl.Route(4096, k, E, torch.zeros(E, **i32), torch.zeros(E + 1, **i32), torch.zeros(4096 * k, **i32))
        experts = torch.zeros(4096 * k, **i32)
        ws = torch.zeros(max(t.ws.numel(), hl.hl_grad_workspace_bytes(), hl.hl_route_workspace_bytes(4096, k, E)),
                         dtype=torch.uint8, device="cuda")
        t.ws = ws
        lose = [t.plan, lambda: hl.hl_route_plan(t.h, route, experts, ws),
                lambda: hl.hl_grad_sq(t.h, hl.GradList([other]), torch.zeros(1, dtype=torch.float64, device="cuda"), ws),
                lambda: hl.hl_embbag_bwd_sgd(t.h, other[:t.n_hot], other[t.n_hot:], t.n_stg, t.codes, t.ptr_d, t.B, t.T,
                                             t.L, None, None, t.B, t.dY, 0.1, ws)]
        for f in lose:
            t.plan()
            t.norm_()
            f()
            with pytest.raises(hl.HotlineError) as e:
                t.clip(w, 1.0, 0.5)
            assert e.value.status == 1
        torch.cuda.synchronize()
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()
