"""One training step of a mixture of experts over the embedding tables, every new
call in its place: rows pooled, tokens sent to experts, weighted back, the
gradients of all of it, one global norm over the experts' weights and the tables,
and the clipped updates; against the same step in 64 bits by automatic
differentiation."""
import math

import numpy as np
import pytest
import torch

from paper_2204_05436_amd import hotline as hl

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("grid", [False, True])
@pytest.mark.parametrize("max_norm", [1e9, 0.5])
@pytest.mark.parametrize("B,T,dim,E,k,capacity,align", [(1, 1, 8, 2, 1, 0, 1), (96, 4, 32, 5, 2, 60, 8),
                                                       (333, 3, 20, 16, 4, 0, 1)])
def test_step(B, T, dim, E, k, capacity, align, max_norm, grid):
    g = torch.Generator().manual_seed(B + dim)
    rows, n_hot, lr = 50, 30, 0.125
    h = hl.hl_create([rows] * T, dim, "f32", T * n_hot)
    try:
        # the tables: the first n_hot rows of each are hot, the others' rows in staging as they come
        hot = (torch.arange(T)[:, None] * rows + torch.arange(n_hot)).view(-1).int().cuda()
        hl.hl_set_hot(h, hot, T * n_hot)
        n_stg, L, n_bags = T * (rows - n_hot), B * T, B * T
        row = torch.randint(0, rows, (B, T), generator=g)
        t = torch.arange(T)
        code = torch.where(row < n_hot, t * n_hot + row, T * n_hot + t * (rows - n_hot) + row - n_hot).view(-1)
        w = torch.randn(T * rows, dim, generator=g).cuda()
        codes, ptr = code.int().cuda(), torch.arange(n_bags + 1, dtype=torch.int32, device="cuda")
        ws = torch.zeros(hl.hl_workspace_bytes(h, L, n_bags, B), dtype=torch.uint8, device="cuda")
        gws = torch.zeros(hl.hl_grad_workspace_bytes(), dtype=torch.uint8, device="cuda")
        # the routing: every bag is a token
        experts = torch.randint(-1, E, (n_bags, k), generator=g, dtype=torch.int32)
        weights = torch.rand(n_bags, k, generator=g).cuda()
        W = (torch.randn(E, dim, dim, generator=g) / math.sqrt(dim)).cuda()
        d_out = torch.randn(n_bags, dim, generator=g).cuda()  # the loss's gradient at the tokens
        if grid:  # small whole numbers: every sum is exact in fp32, in any order
            whole = lambda v, m: torch.randint(-m, m + 1, v.shape, generator=g).float().cuda()
            w, weights, W, d_out = whole(w, 2), whole(weights, 2), whole(W, 1), whole(d_out, 1)
        i32 = dict(dtype=torch.int32, device="cuda")
        n_rows = hl.hl_route_rows(n_bags, k, E, capacity, align)
        counts, offsets = torch.zeros(E, **i32), torch.zeros(E + 1, **i32)
        pos, order = torch.zeros(n_bags * k, **i32), torch.zeros(n_rows, **i32)
        route = hl.Route(n_bags, k, E, counts, offsets, pos, order, capacity, align)
        rws = torch.zeros(max(1, hl.hl_route_workspace_bytes(n_bags, k, E)), dtype=torch.uint8, device="cuda")
        f32 = dict(dtype=torch.float32, device="cuda")
        x, y = torch.zeros(n_bags, dim, **f32), torch.zeros(n_bags, dim, **f32)
        xe, dye = torch.zeros(n_rows, dim, **f32), torch.zeros(n_rows, dim, **f32)
        ye, dxe = torch.zeros(n_rows, dim, **f32), torch.zeros(n_rows, dim, **f32)
        dw, dx, dW = torch.zeros_like(weights), torch.zeros_like(x), torch.zeros_like(W)
        sq, norm = torch.zeros(2, dtype=torch.float64, device="cuda"), torch.zeros(1, **f32)

        hl.hl_embbag_fwd_plan(h, w[:T * n_hot], w[T * n_hot:], n_stg, codes, ptr, B, T, L, x, ws)
        hl.hl_route_plan(h, route, experts.cuda(), rws)
        hl.hl_route_gather(h, route, x, xe)
        at = offsets.tolist()
        blocks = [slice(at[e], at[e + 1]) for e in range(E)]
        for e, b in enumerate(blocks):  # the experts' products, over whole blocks, padding rows included
            ye[b] = xe[b] @ W[e]
        hl.hl_route_combine(h, route, ye, weights, y)
        hl.hl_route_combine_bwd(h, route, d_out, ye, weights, dye, dw)
        for e, b in enumerate(blocks):
            dW[e] = xe[b].t() @ dye[b]
            dxe[b] = dye[b] @ W[e].t()
        hl.hl_route_gather_bwd(h, route, dxe, dx)
        hl.hl_embbag_bwd_norm(h, n_stg, B, T, L, dx, sq[1:], ws)
        grads = hl.GradList([dW, dw])
        hl.hl_grad_sq(h, grads, sq, gws)
        before = (dW.clone(), dw.clone())
        hl.hl_grad_clip(h, grads, sq, max_norm, norm)
        new = w.clone()
        hl.hl_embbag_bwd_clip(h, new[:T * n_hot], new[T * n_hot:], n_stg, B, T, L, sq, max_norm, lr, ws)
        assert hl.hl_last_device_error(h) == 0

        # the same in 64 bits
        w6, W6, g6 = (v.double().cpu().requires_grad_() for v in (w, W, weights))
        x6 = w6[code]
        seen = {e: 0 for e in range(E)}
        out = []
        for b in range(n_bags):
            s = 0.0 * x6[b]  # (a token without an expert depends on nothing)
            for j in range(k):
                e = int(experts[b, j])
                if e < 0:
                    continue
                seen[e] += 1
                if not capacity or seen[e] <= capacity:
                    s = s + g6[b, j] * (x6[b] @ W6[e])
            out.append(s)
        y6 = torch.stack(out)
        got = torch.autograd.grad((y6 * d_out.double().cpu()).sum(), (w6, W6, g6), allow_unused=True)
        gw, gW, gg = (torch.zeros_like(v) if d is None else d for v, d in zip((w6, W6, g6), got))
        n6 = math.sqrt(float(sum(v.square().sum() for v in (gw, gW, gg))))
        c = 1.0 if n6 <= max_norm else max_norm / n6
        if grid:
            # |x W| <= 2 dim, the gradients at most 2 k dim n_bags: below 2^24
            assert 2 * k * dim * n_bags < 2 ** 24 and 4 * dim * dim < 2 ** 24
            assert torch.equal(y.double().cpu(), y6.detach())
            assert torch.equal(before[0].double().cpu(), gW) and torch.equal(before[1].double().cpu(), gg)
            assert abs(float(norm) - n6) <= 2 * U * n6
            for got, ref in ((dW, gW), (dw, gg)):
                assert bool(((got.double().cpu() - c * ref).abs() <= 3 * U * c * ref.abs()).all())
            step = lr * c * gw  # (the factor, the product and the difference are rounded)
            ref = w6.detach() - step
            assert bool(((new.double().cpu() - ref).abs() <= 4 * U * step.abs() + U * ref.abs() * (1 + U)).all())
            return
        # every value is a chain of at most four fp32 sums of up to n terms, n U of the terms' size each (the matrix
        # products' sums in any order); sizes by the same chain with absolute values, at most `size` of the largest
        n = 2 * (max(dim, n_bags) + k + B + 16)

        def near(a, ref, size):
            return bool(((a.double().cpu() - ref).abs() <= 4 * n * U * size).all())

        A = lambda v: v.detach().abs().double().cpu()
        kept = (pos.view(n_bags, k) >= 0).double().cpu()
        top = A(W).sum((1, 2)).max() * max(1.0, float(A(w).max())) * max(1.0, float(A(d_out).max())) * k
        assert near(y, y6.detach(), top)
        assert near(before[0], gW, n_bags * k * float(A(w).max()) * float(A(d_out).max()))
        assert near(before[1], gg, dim * top)
        assert bool((dw.cpu()[kept == 0] == 0).all())
        rel = 4 * n * U * (1 + dim * float(top) * n_bags * k / max(n6, 1e-30))
        assert abs(float(norm) - n6) <= rel * n6 + 2 * U * n6
        assert near(dW, c * gW, n_bags * k * float(A(w).max()) * float(A(d_out).max()) + rel)
        assert near(new, w6.detach() - lr * c * gw, float(A(w).max()) + lr * n_bags * float(top) * (1 + rel))
    finally:
        h.close()
