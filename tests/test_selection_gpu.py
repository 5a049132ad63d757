"""The backward's calls over the first samples of a mini-batch (no list: samples 0 .. n_sel_max - 1) against plain sums
in 64 bits, and bit for bit against the same samples as a list: the one-call update, with and without a workspace, the
plan with the update, and the plan with the norm and the clipped update; and over no sample at all."""
import math

import numpy as np
import pytest
import torch

from paper_2204_05436_amd import hotline as hl
from test_clip_gpu import Tables, U

pytestmark = pytest.mark.gpu

LR = 0.5


def sgd(t, w, ids, n_sel, n_dev=None):
    hl.hl_embbag_bwd_sgd(t.h, w[:t.n_hot], w[t.n_hot:], t.n_stg, t.codes, t.ptr_d, t.B, t.T, t.L, ids, n_dev, n_sel,
                         t.dY, LR, t.ws)


def noalloc(t, w, ids, n_sel, n_dev=None):
    hl.hl_embbag_bwd_sgd_noalloc(t.h, w[:t.n_hot], w[t.n_hot:], t.n_stg, t.codes, t.ptr_d, t.B, t.T, t.L, ids, n_dev,
                                 n_sel, t.dY, LR)


def plan(t, ids, n_sel, n_dev=None):
    hl.hl_embbag_bwd_plan(t.h, t.n_stg, t.codes, t.ptr_d, t.B, t.T, t.L, ids, n_dev, n_sel, t.ws)


def apply(t, w, ids, n_sel, n_dev=None):
    plan(t, ids, n_sel, n_dev)
    t.apply(w, LR)


def clip(t, w, ids, n_sel, n_dev=None):
    plan(t, ids, n_sel, n_dev)
    t.norm_()
    t.clip(w, math.inf, LR)


FORMS = [sgd, noalloc, apply, clip]


@pytest.mark.parametrize("dt,dim,bag", [("f32", 64, 0.0), ("f32", 3, 2.5), ("bf16", 40, 2.5), ("bf16", 16, 0.0)])
@pytest.mark.parametrize("n_sel", [1, 67, 199, 200])
def test_first_samples(dt, dim, bag, n_sel):
    t = Tables(4, 300, dim, dt, 200, bag, seed=7)
    try:
        G, A, n = t.sums(np.arange(n_sel))
        off = n[:, None] * U * A  # an fp32 sum of n terms is off by (n - 1) U of their sizes at most
        ref = t.w.double() - LR * G
        # the sum, the product with the rate, the difference, the row's rounding
        f = torch.finfo(t.w.dtype)
        tol = (LR * off + 4 * U * (LR * (G.abs() + off) + t.w.double().abs()) + f.eps / 2 * ref.abs()) * (1 + f.eps)
        ids = torch.arange(n_sel, dtype=torch.int32, device="cuda")
        for form in FORMS:
            a, b = t.w.clone(), t.w.clone()
            form(t, a, None, n_sel)
            assert bool(((a.double() - ref).abs() <= tol).all()), form.__name__
            assert torch.equal(a[n == 0], t.w[n == 0]), form.__name__
            if n_sel < t.B:  # (a whole one-hot mini-batch is grouped table by table: other tiles)
                form(t, b, ids, n_sel)
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), form.__name__
        want, slack = float(G.square().sum()), float((2 * G.abs() * off + off * off).sum())
        assert abs(float(t.sq) - want) <= slack + 2.0 ** -39 * want
        assert hl.hl_last_device_error(t.h) == 0
        if n_sel == t.B:
            return
        plan(t, None, n_sel)
        keys, bags = (torch.zeros(t.L, dtype=torch.int32, device="cuda") for _ in range(2))
        hl.hl_embbag_bwd_grouping(t.h, *t.shape(), t.ws, keys, bags)
        take = t.bag // t.T < n_sel
        by_row = np.argsort(t.row[take], kind="stable")
        m = int(take.sum())
        assert np.array_equal(keys[:m].cpu().numpy(), t.row[take][by_row]) and bool((keys[m:] == -1).all())
        assert np.array_equal(bags[:m].cpu().numpy(), t.bag[take][by_row])
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()


@pytest.mark.parametrize("dt,dim,bag", [("f32", 64, 0.0), ("bf16", 40, 2.5)])
@pytest.mark.parametrize("how", ["none", "no list", "device count"])
def test_no_samples(dt, dim, bag, how):
    """A selection of no sample of a mini-batch with lookups: no row changes, and the norm is zero."""
    t = Tables(3, 90, dim, dt, 50, bag, seed=8)
    try:
        i32 = dict(dtype=torch.int32, device="cuda")
        ids = None if how == "none" else torch.zeros(4, **i32)
        n_sel, n_dev = (4, torch.zeros(1, **i32)) if how == "device count" else (0, None)
        w = t.w.clone()
        for form in FORMS:
            t.sq.fill_(7.0)
            t.norm.fill_(7.0)
            form(t, w, ids, n_sel, n_dev)
            assert torch.equal(w, t.w), form.__name__
        assert float(t.sq) == 0 and float(t.norm) == 0
        plan(t, ids, n_sel, n_dev)
        for part in (1, 2):
            hl.hl_embbag_bwd_apply_part(t.h, w[:t.n_hot], w[t.n_hot:], *t.shape(), t.dY, LR, part, t.ws)
        keys, bags = (torch.zeros(t.L, **i32) for _ in range(2))
        hl.hl_embbag_bwd_grouping(t.h, *t.shape(), t.ws, keys, bags)
        assert bool((keys == -1).all()) and torch.equal(w, t.w)
        # other sizes than the plan's are refused as ever
        for f in (lambda: hl.hl_embbag_bwd_apply(t.h, w[:t.n_hot], w[t.n_hot:], t.n_stg, t.B, t.T, t.L - 1, t.dY, LR, t.ws),
                  lambda: hl.hl_embbag_bwd_norm(t.h, t.n_stg, t.B, t.T, t.L - 1, t.dY, t.sq, t.ws)):
            with pytest.raises(hl.HotlineError):
                f()
        # the next plan on this workspace groups as ever
        G, _, n = t.sums()
        apply(t, w, None, t.B)
        assert not torch.equal(w, t.w) and torch.equal(w[n == 0], t.w[n == 0])
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()
