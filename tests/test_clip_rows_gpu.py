"""The clipped table update against the plain one where runs of equal rows span many tiles and their sums cancel to
rounding errors, so that another order of the additions shows: bit for bit where both calls take as many elements per
lane, within the bound of an fp32 sum where they do not.  Which calls may come between the norm and the update, codes
that name no row, the longest rows, and mini-batches of hot or of staging rows alone."""
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


def held_to_sums(t, row, bag, n_rows, plan, norm, clip, apply, w0, n_hot):
    """Norm and clipped update of the lookups (row, bag) against sums in 64 bits, and bit for bit the plain update where
    the rows' addresses promise it."""
    row, bag = torch.from_numpy(row).cuda(), torch.from_numpy(bag).cuda()
    G = torch.zeros(n_rows, t.dY.shape[1], dtype=torch.float64, device="cuda")
    A, n = torch.zeros_like(G), torch.zeros(n_rows, dtype=torch.float64, device="cuda")
    d = t.dY.double()[bag]
    G, A = G.index_add(0, row, d), A.index_add(0, row, d.abs())
    n = n.index_add(0, row, torch.ones(row.numel(), dtype=torch.float64, device="cuda"))
    off = n[:, None] * U * A
    plan()
    norm()
    want = float(G.square().sum())
    assert abs(float(t.sq) - want) <= float((2 * G.abs() * off + off * off).sum()) + 2.0 ** -39 * want
    m = float(np.float32(math.sqrt(want) / 5))
    c = np.float32(m / math.sqrt(float(t.sq)))
    a, b = w0.clone(), w0.clone()
    clip(a, m)
    apply(b, float(np.float32(0.5) * c))
    wide = 32 if w0.dtype is torch.bfloat16 and w0.shape[1] % 8 == 0 else 16
    if n_hot * w0.shape[1] * w0.element_size() % wide == 0:
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    f = torch.finfo(w0.dtype)
    ref = w0.double() - 0.5 * float(c) * G
    tol = 0.5 * float(c) * off + 4 * U * (0.5 * float(c) * (G.abs() + off) + w0.double().abs()) + f.eps / 2 * ref.abs()
    assert bool(((a.double() - ref).abs() <= tol * (1 + f.eps)).all())
    assert torch.equal(a[n == 0], w0[n == 0]) and not torch.equal(a, w0)


@pytest.mark.parametrize("bag", [0.0, 2.0])
@pytest.mark.parametrize("dt,dim", [("f32", 64), ("bf16", 24)])
def test_codes_of_no_row(dt, dim, bag):
    """Lookups whose code names no row are reported and have no part in the norm or the update."""
    t = Tables(3, 100, dim, dt, 300, bag, seed=6)
    try:
        bad = np.random.RandomState(1).rand(t.L) < 0.1
        codes = t.row.astype(np.int32)
        codes[bad] = np.resize(np.array([-1, -(2 ** 31), t.n_hot + t.n_stg, 2 ** 31 - 1], np.int32), int(bad.sum()))
        t.codes.copy_(torch.from_numpy(codes))
        held_to_sums(t, t.row[~bad], t.bag[~bad], t.w.shape[0], t.plan, t.norm_, lambda w, m: t.clip(w, m, 0.5), t.apply,
                     t.w, t.n_hot)
        assert hl.hl_last_device_error(t.h) == hl.DEVERR["BAD_CODE"]
    finally:
        t.h.close()


@pytest.mark.parametrize("dim,dt", [(8192, "f32"), (8192, "bf16"), (4100, "f32"), (8190, "bf16")])
def test_longest_rows(dim, dt):
    t = Tables(2, 12, dim, dt, 90, 3.0, seed=2, hot=0.5)
    try:
        held_to_sums(t, t.row, t.bag, t.w.shape[0], t.plan, t.norm_, lambda w, m: t.clip(w, m, 0.5), t.apply, t.w,
                     t.n_hot)
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()


@pytest.mark.parametrize("dt,dim", [("f32", 16), ("bf16", 8)])
@pytest.mark.parametrize("hot", [False, True])
def test_rows_of_one_kind(hot, dt, dim):
    """Only staging rows (no hot set, no hot cache), or only hot rows (no staging buffer)."""
    B, T, rows = 70, 2, 15
    k_cap = T * rows
    h = hl.hl_create([rows] * T, dim, dt, k_cap)
    try:
        if hot:
            hl.hl_set_hot(h, torch.arange(k_cap, dtype=torch.int32, device="cuda"), k_cap)
        g = np.random.RandomState(3)
        row = (g.randint(0, rows, (B, T)) + np.arange(T) * rows).reshape(-1)
        codes = torch.from_numpy((row if hot else row + k_cap).astype(np.int32)).cuda()
        L, n_stg = B * T, 0 if hot else k_cap
        ptr = torch.arange(L + 1, dtype=torch.int32, device="cuda")
        ws = torch.zeros(hl.hl_workspace_bytes(h, L, L, B), dtype=torch.uint8, device="cuda")

        class t:
            dY = torch.randn(L, dim, generator=torch.Generator().manual_seed(4)).cuda()
            sq, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")

        kind = lambda w: (w, None) if hot else (None, w)
        w0 = torch.randn(k_cap, dim, generator=torch.Generator().manual_seed(5)).to(
            torch.float32 if dt == "f32" else torch.bfloat16).cuda()
        held_to_sums(t, row, np.arange(L), k_cap,
                     lambda: hl.hl_embbag_bwd_plan(h, n_stg, codes, ptr, B, T, L, None, None, B, ws),
                     lambda: hl.hl_embbag_bwd_norm(h, n_stg, B, T, L, t.dY, t.sq, ws),
                     lambda w, m: hl.hl_embbag_bwd_clip(h, *kind(w), n_stg, B, T, L, t.sq, m, 0.5, ws, t.norm),
                     lambda w, lr: hl.hl_embbag_bwd_apply(h, *kind(w), n_stg, B, T, L, t.dY, lr, ws), w0, 0)
        assert hl.hl_last_device_error(h) == 0
    finally:
        h.close()
