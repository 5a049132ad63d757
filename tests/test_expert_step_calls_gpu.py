"""The training step of a mixture of experts over the embedding tables, call by call: each output against the same
formula in 64 bits on the call's own fp32 inputs, element by element, with bounds that count that call's roundings (and
that no zero, unclipped or unweighted output would pass: `near` asks for it)."""
import math

import pytest
import torch

from paper_2204_05436_amd import hotline as hl

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32, relative


def near(a, ref, tol, what):
    a, ref, tol = a.double().cpu(), ref.cpu(), tol.cpu()
    size = float(ref.abs().max())
    assert size > 0, what + ": nothing to compare"
    assert float(tol.max()) <= 2.0 ** -12 * size, what + ": the bound says nothing"
    bad = (a - ref).abs() - tol
    assert bool((bad <= 0).all()), f"{what}: {float(bad.max())} past the bound, values up to {size}"


@pytest.mark.parametrize("max_norm", [1e9, 0.5])
@pytest.mark.parametrize("B,T,dim,E,k,capacity,align", [(1, 1, 8, 2, 1, 0, 1), (96, 4, 32, 5, 2, 60, 8),
                                                       (333, 3, 20, 16, 4, 0, 1), (50, 2, 300, 3, 1, 0, 4)])
def test_step(B, T, dim, E, k, capacity, align, max_norm):
    g = torch.Generator().manual_seed(B + dim)
    rows, n_hot, lr = 50, 30, 0.125
    h = hl.hl_create([rows] * T, dim, "f32", T * n_hot)
    try:
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
        experts = torch.randint(-1, E, (n_bags, k), generator=g, dtype=torch.int32)
        if n_bags == 1:
            experts.fill_(E - 1)  # (the one token is kept)
        weights = (torch.rand(n_bags, k, generator=g) + 0.25).cuda()
        W = (torch.randn(E, dim, dim, generator=g) / math.sqrt(dim)).cuda()
        d_out = torch.randn(n_bags, dim, generator=g).cuda()
        i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
        n_rows = hl.hl_route_rows(n_bags, k, E, capacity, align)
        counts, offsets = torch.zeros(E, **i32), torch.zeros(E + 1, **i32)
        pos, order = torch.zeros(n_bags * k, **i32), torch.zeros(n_rows, **i32)
        route = hl.Route(n_bags, k, E, counts, offsets, pos, order, capacity, align)
        rws = torch.zeros(max(1, hl.hl_route_workspace_bytes(n_bags, k, E)), dtype=torch.uint8, device="cuda")
        x, y = torch.zeros(n_bags, dim, **f32), torch.zeros(n_bags, dim, **f32)
        xe, dye = torch.zeros(n_rows, dim, **f32), torch.zeros(n_rows, dim, **f32)
        ye, dxe = torch.zeros(n_rows, dim, **f32), torch.zeros(n_rows, dim, **f32)
        dw, dx, dW = torch.full_like(weights, 9.0), torch.zeros_like(x), torch.zeros_like(W)
        sq, norm = torch.zeros(2, dtype=torch.float64, device="cuda"), torch.zeros(1, **f32)

        hl.hl_embbag_fwd_plan(h, w[:T * n_hot], w[T * n_hot:], n_stg, codes, ptr, B, T, L, x, ws)
        hl.hl_route_plan(h, route, experts.cuda(), rws)
        hl.hl_route_gather(h, route, x, xe)
        at = offsets.tolist()
        blocks = [slice(at[e], at[e + 1]) for e in range(E)]
        for e, b in enumerate(blocks):
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
        before = dW.clone(), dw.clone()
        hl.hl_grad_clip(h, grads, sq, max_norm, norm)
        new = w.clone()
        hl.hl_embbag_bwd_clip(h, new[:T * n_hot], new[T * n_hot:], n_stg, B, T, L, sq, max_norm, lr, ws)
        assert hl.hl_last_device_error(h) == 0

        # the plan: which assignment is in which row
        seen, want = [0] * E, torch.full((n_bags * k,), -1)
        for a, e in enumerate(experts.view(-1).tolist()):
            if e >= 0:
                if not capacity or seen[e] < capacity:
                    want[a] = at[e] + seen[e]
                seen[e] += 1
        assert torch.equal(pos.cpu().long(), want)
        kept = want >= 0
        assert bool(kept.any()) and (not capacity or max(seen) > capacity)  # (some are kept, some dropped)
        a = kept.nonzero().view(-1)
        p, tok = want[a].cuda(), (a // k).cuda()
        a = a.cuda()
        D = lambda v: v.double()
        wa = D(weights.view(-1)[a])[:, None]

        assert torch.equal(x, w[code.cuda()])                  # one row per bag
        assert torch.equal(xe[p], x[tok])                      # copies
        used = torch.zeros(n_rows, dtype=torch.bool, device="cuda")
        used[p] = True
        pad = ~used
        pad[at[E]:] = False                                    # (rows behind the last block are not written)
        assert not bool(xe[pad].any()) and not bool(dye[pad].any())
        zero = torch.zeros(n_bags, dim, dtype=torch.float64, device="cuda")
        add = lambda v: zero.index_add(0, tok, v)
        # a sum of k products by fused multiply-adds: k roundings; a sum of k rows: as many
        near(y, add(wa * D(ye[p])), (k + 1) * U * add((wa * D(ye[p])).abs()), "combine")
        near(dx, add(D(dxe[p])), (k + 1) * U * add(D(dxe[p]).abs()), "gather_bwd")
        near(dye[p], wa * D(d_out[tok]), U * (wa * D(d_out[tok])).abs(), "combine_bwd rows")
        # dim fused multiply-adds and the lanes' sums, at most dim + 10 roundings of any term
        prod = D(d_out[tok]) * D(ye[p])
        near(before[1].view(-1)[a], prod.sum(1), (dim + 10) * U * prod.abs().sum(1), "combine_bwd weights")
        dropped = (~kept).nonzero().view(-1).cuda()
        assert not bool(before[1].view(-1)[dropped].any())
        # the tables' gradient: n lookups of a row are n - 1 roundings
        G = torch.zeros(T * rows, dim, dtype=torch.float64, device="cuda")
        A, c6 = G.clone(), code.cuda()
        n = torch.zeros(T * rows, dtype=torch.float64, device="cuda").index_add(0, c6, torch.ones(L, dtype=torch.float64, device="cuda"))
        G, A = G.index_add(0, c6, D(dx)), A.index_add(0, c6, D(dx).abs())
        off = (n[:, None] - 1).clamp(min=0) * (1 + 2.0 ** -10) * U * A
        s = sq.tolist()
        dense, table = float(sum(D(v).square().sum() for v in before)), float(G.square().sum())
        assert abs(s[0] - dense) <= 2.0 ** -39 * dense and s[0] > 0
        slack = float((2 * G.abs() * off + off * off).sum())
        assert slack <= 2.0 ** -12 * table and abs(s[1] - table) <= slack + 2.0 ** -39 * table
        full = math.sqrt(s[0] + s[1])
        assert abs(float(norm) - full) <= 2 * U * full
        assert 0.5 < full < 1e9  # (one of the two bounds clips, the other does not)
        c = min(1.0, max_norm / full)
        for got, src, what in ((dW, before[0], "clipped experts"), (dw, before[1], "clipped weights")):
            if c == 1.0:
                assert torch.equal(got, src)
            # the factor and the product, each rounded
            near(got, c * D(src), (2 * U + U * U) * c * D(src).abs(), what)
        ref = D(w) - lr * c * G
        step = new.double() - D(w)
        # the sum, the factor, the rate's product, the product, the difference
        tol = lr * c * off + 4 * U * lr * c * (G.abs() + off) + U * (1 + 2.0 ** -10) * ref.abs()
        assert bool(((new.double() - ref).abs() <= tol).all())
        assert torch.equal(new[n == 0], w[n == 0])
        # the bound against the step itself (the rows are larger than it): most of what moved is told apart from zero
        big = lr * c * G.abs() > 16 * tol
        assert float(big.double().mean()) > 0.25 * float((G != 0).double().mean()) > 0
        assert bool((step[big] != 0).all())
    finally:
        h.close()
