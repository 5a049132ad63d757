"""Routing to experts on the GPU: the plan's integers against a loop over the
experts, and the row movements with their gradients against plain sums in 64
bits, at the sizes where the kernels change form, with padding ids, capacities,
block alignments, strides and addresses that divide nothing."""
import numpy as np
import pytest
import torch

from paper_2204_05436_amd import hotline as hl

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24  # half a step of fp32, relative


@pytest.fixture(scope="module")
def h():
    x = hl.hl_create([1], 1, "f32", 1)
    yield x
    x.close()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def least(dtype):
    """Half a step of the type's subnormal numbers."""
    f = torch.finfo(dtype)
    return f.smallest_normal * f.eps / 2


def plan_ref(experts, n_experts, capacity, align, n_rows):
    e = np.asarray(experts).reshape(-1)
    counts, offsets = np.zeros(n_experts, np.int64), np.zeros(n_experts + 1, np.int64)
    pos, order = np.full(e.size, -1, np.int64), np.full(n_rows, -7, np.int64)
    by_expert = np.argsort(np.where((e < 0) | (e >= n_experts), n_experts, e), kind="stable")
    first = np.searchsorted(np.sort(np.where((e < 0) | (e >= n_experts), n_experts, e)), np.arange(n_experts + 1))
    for x in range(n_experts):
        mine = by_expert[first[x]:first[x + 1]]
        mine = mine[:capacity] if capacity else mine
        counts[x] = mine.size
        offsets[x + 1] = offsets[x] + -(-mine.size // align) * align
        order[offsets[x]:offsets[x + 1]] = -1
        order[offsets[x]:offsets[x] + mine.size] = mine
        pos[mine] = offsets[x] + np.arange(mine.size)
    return counts, offsets, pos, order


class Plan:
    def __init__(self, h, experts, n_experts, capacity=0, align=1, extra=3, order=True, stream=None):
        t, k = experts.shape
        i32 = dict(dtype=torch.int32, device="cuda")
        self.n_rows = hl.hl_route_rows(t, k, n_experts, capacity, align) + extra
        self.counts, self.offsets = torch.full((n_experts,), -9, **i32), torch.full((n_experts + 1,), -9, **i32)
        self.pos = torch.full((t * k,), -9, **i32)
        self.order = torch.full((self.n_rows,), -7, **i32) if order else None
        self.route = hl.Route(t, k, n_experts, self.counts, self.offsets, self.pos, self.order, capacity, align,
                              n_rows=self.n_rows)
        self.ws = torch.zeros(max(1, hl.hl_route_workspace_bytes(t, k, n_experts)), dtype=torch.uint8, device="cuda")
        self.experts = experts.cuda()
        self.args = (n_experts, capacity, align)
        hl.hl_route_plan(h, self.route, self.experts, self.ws, stream=stream)

    def check(self):
        counts, offsets, pos, order = plan_ref(self.experts.cpu().numpy(), *self.args, self.n_rows)
        assert np.array_equal(self.counts.cpu().numpy(), counts)
        assert np.array_equal(self.offsets.cpu().numpy(), offsets)
        assert np.array_equal(self.pos.cpu().numpy(), pos)
        if self.order is not None:
            assert np.array_equal(self.order.cpu().numpy(), order)


def ids(seed, t, k, n_experts, drop=0.0, one=False):
    g = np.random.RandomState(seed)
    e = g.zipf(1.3, (t, k)) % n_experts if not one else np.full((t, k), n_experts - 1)
    e[g.rand(t, k) < drop] = -1
    return torch.from_numpy(e.astype(np.int32))


@pytest.mark.parametrize("t,k,n_experts,capacity,align,drop", [
    (0, 2, 5, 0, 4, 0), (1, 1, 1, 0, 1, 0), (1, 8, 256, 0, 1, 0), (1, 3, 4, 1, 16, 0), (63, 1, 2, 0, 1, 0.5),
    (64, 1, 64, 0, 1, 0), (65, 5, 37, 4, 3, 0.2), (1024, 1, 8, 0, 1, 0), (1025, 1, 8, 100, 128, 0.1),
    (2049, 2, 1000, 0, 1, 0), (1024, 8, 1024, 0, 16, 0.1), (8193, 1, 3, 0, 1, 0), (4096, 8, 64, 0, 16, 0),
    (4096, 8, 64, 520, 1, 0.3), (16385, 8, 1024, 7, 5, 0), (70001, 8, 129, 0, 64, 0), (300007, 7, 8, 0, 1, 0.01),
    (1 << 18, 9, 33, 1000, 1, 0.05), (9000, 1, 5, 0, 7, 1.0), (4096, 1, 1024, 0, 1, 0), (4097, 1, 1024, 3, 2, 0),
    (8192, 1, 1024, 0, 1, 0.1), (8193, 1, 1023, 0, 1, 0.1), (262144, 1, 31, 0, 8, 0), (262145, 1, 33, 0, 8, 0)])
def test_plan(h, t, k, n_experts, capacity, align, drop):
    Plan(h, ids(t + k, t, k, n_experts, drop), n_experts, capacity, align).check()
    assert hl.hl_last_device_error(h) == 0


@pytest.mark.parametrize("t", [5, 5000, 40000])
def test_plan_one_expert_takes_all(h, t):
    Plan(h, ids(0, t, 2, 6, one=True), 6, align=4).check()
    Plan(h, ids(0, t, 2, 6, one=True), 6, capacity=t, align=4, order=False).check()
    assert hl.hl_last_device_error(h) == 0


@pytest.mark.parametrize("t", [7, 30000])
def test_plan_bad_ids(h, t):
    """Ids outside [-1, n_experts) are reported and not kept."""
    e = ids(3, t, 2, 9)
    e[0, 1], e[t // 2, 0], e[t - 1, 1] = 9, -2, 2 ** 31 - 1
    p = Plan(h, e, 9)
    assert hl.hl_last_device_error(h) == hl.DEVERR["OUT_OF_RANGE"]
    p.check()


def rows_of(n, dim, dtype, seed, stride=None, shift=0, fill=None):
    """[n, dim] rows `stride` elements apart, the first `shift` elements into its buffer; and the buffer."""
    stride = stride or dim
    buf = torch.full((n * stride + shift + 8,), 3.0, dtype=dtype, device="cuda")
    v = buf[shift:shift + n * stride].view(n, stride)[:, :dim]
    if fill is None:
        v.copy_(torch.randn(n, dim, generator=torch.Generator().manual_seed(seed)).to(dtype))
    else:
        v.fill_(fill)
    return v, buf


def untouched(v, buf, before):
    """Everything of buf outside the rows v is as it was."""
    keep = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(keep, v.shape, v.stride(), v.storage_offset()).fill_(False)
    assert torch.equal(buf[keep].view(torch.uint8), before[keep].view(torch.uint8))


SHAPES = [  # tokens, k, experts, dim, capacity, align, drop, spare elements per row, first element
    (1, 1, 1, 1, 0, 1, 0, 0, 0), (1, 2, 8, 1024, 0, 1, 0, 0, 0), (3, 8, 16, 7, 0, 4, 0.3, 1, 1),
    (65, 3, 5, 64, 20, 1, 0.1, 0, 0), (130, 9, 20, 513, 0, 16, 0.2, 3, 1), (257, 2, 4, 96, 0, 8, 0, 8, 4),
    (40, 17, 33, 2050, 0, 2, 0.1, 0, 3), (2001, 4, 12, 33, 300, 3, 0.5, 0, 0), (33, 2, 7, 4096, 0, 1, 1.0, 0, 0),
    (300, 8, 64, 520, 0, 1, 0, 0, 0), (5000, 2, 6, 256, 0, 1, 0.05, 0, 0), (1200, 1, 3, 1280, 0, 128, 0, 16, 8)]


def at_tokens(plan, t, k):
    """(assignment, token, row) of every kept assignment."""
    p = plan.pos.long()
    a = (p >= 0).nonzero().view(-1)
    return a, torch.div(a, k, rounding_mode="floor"), p[a]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_rows(h, shape, dt):
    t, k, E, dim, cap, align, drop, slack, shift = shape
    dtype, seed = DT[dt], t + dim
    p = Plan(h, ids(seed, t, k, E, drop), E, cap, align)
    p.check()
    a, tok, row = at_tokens(p, t, k)
    used = torch.zeros(p.n_rows, dtype=torch.bool, device="cuda")
    used[row] = True
    total = int(p.offsets[-1])
    padding = ~used
    padding[total:] = False
    stride = dim + slack
    w = torch.randn(t, k, generator=torch.Generator().manual_seed(5)).cuda()
    w_in = w.clone().view(-1)
    w_in[(p.pos < 0)] = float("nan")  # weights of dropped assignments are never used
    # gather: the same values at the experts' rows, zeros in the padding, nothing behind
    x, _ = rows_of(t, dim, dtype, 1, stride, shift)
    rows, buf = rows_of(p.n_rows, dim, dtype, 0, stride, shift, fill=5.0)
    before = buf.clone()
    hl.hl_route_gather(h, p.route, x, rows)
    want = torch.full_like(rows, 5.0)
    want[padding] = 0
    want[row] = x[tok]
    assert torch.equal(rows, want)
    untouched(rows, buf, before)
    # combine: rows that no assignment has hold NaN, which must not show
    y, _ = rows_of(p.n_rows, dim, dtype, 2, stride, shift)
    y[~used] = float("nan")
    out, buf = rows_of(t, dim, dtype, 0, stride, shift, fill=5.0)
    before = buf.clone()
    for weights in (w_in, None):
        hl.hl_route_combine(h, p.route, y, weights, out)
        ww = w.view(-1)[a].double() if weights is not None else torch.ones(a.numel(), dtype=torch.float64, device="cuda")
        terms = y[row].double() * ww[:, None]
        ref = torch.zeros(t, dim, dtype=torch.float64, device="cuda").index_add_(0, tok, terms)
        size = torch.zeros_like(ref).index_add_(0, tok, terms.abs())
        # k products and sums, each off by U of at most `size` (a product's rounding where it is not fused), then the
        # type's rounding
        tol = (2 * k * U * size) * (1 + half_step(dtype)) + half_step(dtype) * ref.abs() + least(dtype)
        assert ((out.double() - ref).abs() <= tol).all()
        untouched(out, buf, before)
    # gather's gradient is combine's sum without weights
    dx, buf = rows_of(t, dim, dtype, 0, stride, shift, fill=5.0)
    hl.hl_route_gather_bwd(h, p.route, y, dx)
    assert torch.equal(dx, out)
    # combine's gradients
    d, _ = rows_of(t, dim, dtype, 3, stride, shift)
    drows, buf = rows_of(p.n_rows, dim, dtype, 0, stride, shift, fill=5.0)
    before = buf.clone()
    dw = torch.full((t, k), 9.0, device="cuda")
    hl.hl_route_combine_bwd(h, p.route, d, y, w_in, drows, dw)
    ref = torch.full((p.n_rows, dim), 5.0, dtype=torch.float64, device="cuda")
    ref[padding] = 0
    ref[row] = d[tok].double() * w.view(-1)[a].double()[:, None]
    tol = (U + half_step(dtype) * (1 + U)) * ref.abs() + least(dtype)
    tol[~used] = 0
    assert ((drows.double() - ref).abs() <= tol).all()
    untouched(drows, buf, before)
    terms = d[tok].double() * y[row].double()
    ref = torch.zeros(t * k, dtype=torch.float64, device="cuda")
    ref[a] = terms.sum(1)
    size = torch.zeros_like(ref)
    size[a] = terms.abs().sum(1)
    # a lane adds up every 64th part of a row or fewer, then lanes and waves are added pairwise
    N = 16 // x.element_size()
    depth = N * -(-dim // (64 * N)) + 10
    assert ((dw.view(-1).double() - ref).abs() <= 2 * depth * U * size).all()
    # without the weights' gradients the rows are not read
    again, _ = rows_of(p.n_rows, dim, dtype, 0, stride, shift, fill=5.0)
    hl.hl_route_combine_bwd(h, p.route, d, None, w_in, again)
    assert torch.equal(again, drows)
    hl.hl_route_combine_bwd(h, p.route, d, None, None, again)
    assert torch.equal(again[row], d[tok])
    assert hl.hl_last_device_error(h) == 0


def test_gradients_by_differences(h):
    """combine's and gather's gradients against central differences of a scalar of their outputs, in fp32: the step
    2^-6 is exact in the inputs' grid of 2^-10, so a difference is off by the sums' rounding alone."""
    t, k, E, dim = 6, 3, 4, 5
    p = Plan(h, ids(1, t, k, E, 0.2), E)
    g = torch.Generator().manual_seed(0)
    grid = lambda *s: (torch.randint(-1024, 1024, s, generator=g).float() / 1024).cuda()
    x, w, d = grid(t, dim), grid(t, k), grid(t, dim)
    rows, out = torch.zeros(p.n_rows, dim, device="cuda"), torch.zeros(t, dim, device="cuda")

    def f(x, w):  # sum of d * combine(gather(x)), in 64 bits
        hl.hl_route_gather(h, p.route, x, rows)
        hl.hl_route_combine(h, p.route, rows, w, out)
        return float((out.double() * d.double()).sum())

    f(x, w)
    drows, dw, dx = torch.zeros_like(rows), torch.zeros_like(w), torch.zeros_like(x)
    hl.hl_route_combine_bwd(h, p.route, d, rows.clone(), w, drows, dw)
    hl.hl_route_gather_bwd(h, p.route, drows, dx)
    step = 2.0 ** -6
    # f is linear in each input; its fp32 sums of 3 terms of at most 1 are off by 6 U each, over t * dim outputs, and
    # the gradients by 10 U of sums of at most 5
    tol = 2 * (6 * U * t * dim) / (2 * step) + 50 * U
    for v, got in ((x, dx), (w, dw)):
        for i in range(v.numel()):
            lo, hi = v.clone(), v.clone()
            lo.view(-1)[i] -= step
            hi.view(-1)[i] += step
            a, b = (f(lo, w), f(hi, w)) if v is x else (f(x, lo), f(x, hi))
            assert abs((b - a) / (2 * step) - float(got.view(-1)[i])) <= tol


def test_bad_places_are_reported(h):
    """pos entries that name no row: reported, not followed."""
    e = ids(2, 50, 2, 4)
    p = Plan(h, e, 4)
    x, rows = torch.randn(50, 24, device="cuda"), torch.zeros(p.n_rows, 24, device="cuda")
    good = p.pos.clone()
    for bad in (p.n_rows, -2, 2 ** 31 - 1):
        p.pos.copy_(good)
        p.pos[17] = bad
        for call in (lambda: hl.hl_route_gather(h, p.route, x, rows),
                     lambda: hl.hl_route_combine(h, p.route, rows, None, x),
                     lambda: hl.hl_route_combine_bwd(h, p.route, x, rows, None, rows.clone(),
                                                     torch.zeros(100, device="cuda"))):
            call()
            assert hl.hl_last_device_error(h) == hl.DEVERR["BAD_CODE"]


def test_far_rows(h):
    """Rows past 2^32 bytes into their buffer: offsets in 64 bits."""
    t, k, E, dim, stride = 20, 1, 2, 200, 1 << 26  # (a stride of 256 MiB)
    e = torch.zeros(t, k, dtype=torch.int32)
    e[::2] = 1
    p = Plan(h, e, E, extra=1)
    p.check()
    n = p.n_rows
    buf = torch.zeros((n - 1) * stride + dim, dtype=torch.float32, device="cuda")
    rows = torch.as_strided(buf, (n, dim), (stride, 1))
    x = torch.randn(t, dim, device="cuda")
    hl.hl_route_gather(h, p.route, x, rows)
    assert torch.equal(rows[p.pos.long()], x)
    out, dw = torch.zeros_like(x), torch.zeros(t, 1, device="cuda")
    hl.hl_route_combine(h, p.route, rows, None, out)
    assert torch.equal(out, x)
    assert hl.hl_last_device_error(h) == 0


def test_many_blocks(h):
    """More blocks than one dimension of a grid is given (2^20): the second one counts."""
    t, dim, E = (1 << 20) + 70_001, 1024, 3
    e = torch.randint(-1, E, (t, 1), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    p = Plan(h, e, E, align=64, order=False)
    p.check()
    x = torch.empty(t, dim, dtype=torch.float32, device="cuda")
    x.copy_(torch.arange(t, dtype=torch.float32, device="cuda")[:, None])  # (every row its number, below 2^24)
    rows = torch.full((p.n_rows, dim), -5.0, device="cuda")
    hl.hl_route_gather(h, p.route, x, rows)
    pos = p.pos.long()
    kept = (pos >= 0).nonzero().view(-1)
    want = torch.full((p.n_rows,), 0.0, device="cuda")
    want[pos[kept]] = kept.float()
    want[int(p.offsets[-1]):] = -5.0
    assert bool((rows == want[:, None]).all())
    hl.hl_route_combine(h, p.route, rows, torch.full((t, 1), 2.0, device="cuda"), x)
    want = torch.zeros(t, device="cuda")
    want[kept] = 2.0 * kept.float()
    assert bool((x == want[:, None]).all())
    dw = torch.full((t, 1), 9.0, device="cuda")
    hl.hl_route_combine_bwd(h, p.route, x, rows, None, rows.new_zeros(rows.shape), dw)
    ref = torch.zeros(t, dtype=torch.float64, device="cuda")
    ref[kept] = 2.0 * kept.double() ** 2 * dim
    assert ((dw.view(-1).double() - ref).abs() <= 2 * (4 * 4 + 10) * U * ref).all()
    assert hl.hl_last_device_error(h) == 0


def test_workspace_of_other_calls():
    """A workspace that other calls use serves the plan too, and serves them afterwards (its header's counters stay)."""
    T, B, L = 2, 3000, 6000
    h = hl.hl_create([500] * T, 8, "f32", 100)
    try:
        hl.hl_set_hot(h, torch.arange(0, 1000, 10, dtype=torch.int32, device="cuda"), 100)
        r = torch.randint(0, 500, (L,), dtype=torch.int32, generator=torch.Generator().manual_seed(3)).cuda()
        ptr = torch.arange(L + 1, dtype=torch.int32, device="cuda")
        t, k, E = 20000, 2, 300
        size = max(hl.hl_workspace_bytes(h, L, L, B), hl.hl_route_workspace_bytes(t, k, E), hl.hl_grad_workspace_bytes())
        ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
        i32 = dict(dtype=torch.int32, device="cuda")
        first = None
        for turn in range(4):
            out = [torch.zeros(n, **i32) for n in (L, L)] + [torch.zeros(B, dtype=torch.uint8, device="cuda")]
            lists = [torch.zeros(n, **i32) for n in (B, B, 2)]
            hl.hl_dispatch(h, r, ptr, B, T, L, *out, *lists, ws)
            assert hl.hl_last_device_error(h) == 0
            got = [x.clone() for x in out + lists]
            first = first or got
            assert all(torch.equal(a, b) for a, b in zip(first, got))
            p = Plan(h, ids(turn, t, k, E), E)
            hl.hl_route_plan(h, p.route, p.experts, ws)
            p.check()
            g = torch.full((300_000 * (1 + 20 * (turn % 2)),), 0.5, device="cuda")  # (few and many blocks)
            sq = torch.zeros(1, dtype=torch.float64, device="cuda")
            hl.hl_grad_sq(h, hl.GradList([g]), sq, ws)
            assert float(sq) == 0.25 * g.numel()
    finally:
        h.close()


def test_refusals(h):
    p = Plan(h, ids(0, 4, 2, 3), 3, align=2)
    r, L = p.route, hl.lib()
    x, rows = torch.zeros(4, 8, device="cuda"), torch.zeros(p.n_rows, 8, device="cuda")

    def status(f, *a):
        with pytest.raises(hl.HotlineError) as e:
            f(*a)
        return e.value.status

    def with_field(**kw):
        q = hl.Route(4, 2, 3, p.counts, p.offsets, p.pos, p.order, 0, 2, n_rows=p.n_rows)
        for name, v in kw.items():
            setattr(q.struct, name, v)
        return q

    for kw, want in [(dict(n_tokens=-1), 1), (dict(k=0), 1), (dict(n_experts=0), 1), (dict(capacity=-1), 1),
                     (dict(align=0), 1), (dict(counts=None), 1), (dict(offsets=None), 1), (dict(pos=None), 1),
                     (dict(n_experts=1025), 5), (dict(n_tokens=1 << 40), 5), (dict(n_rows=1), 3),
                     (dict(align=2 ** 31 - 1), 5)]:
        q = with_field(**kw)
        assert L.hl_route_plan(h.ptr, hl.C.byref(q.struct), p.experts.data_ptr(), None, 0, None) == want, kw
        assert L.hl_route_gather(h.ptr, hl.C.byref(q.struct), 0, 8, x.data_ptr(), 8, rows.data_ptr(), 8, None) == want
    S, X, R = hl.C.byref(r.struct), x.data_ptr(), rows.data_ptr()
    assert L.hl_route_gather(h.ptr, S, 0, (1 << 20) + 1, X, 1 << 21, R, 1 << 21, None) == 5
    q = with_field(n_tokens=1 << 28, k=1, n_rows=1 << 29)
    assert L.hl_route_gather(h.ptr, hl.C.byref(q.struct), 0, 1 << 20, X, 1 << 20, R, 1 << 20, None) == 5
    assert L.hl_route_plan(h.ptr, S, None, None, 0, None) == 1
    assert L.hl_route_plan(h.ptr, None, p.experts.data_ptr(), None, 0, None) == 1
    for args in [(3, 8, X, 8, R, 8), (-1, 8, X, 8, R, 8), (0, 0, X, 8, R, 8), (0, 8, X, 7, R, 8), (0, 8, X, 8, R, 7),
                 (0, 8, None, 8, R, 8), (0, 8, X, 8, None, 8), (0, 8, X + 2, 8, R, 8), (1, 8, X, 8, R + 1, 8)]:
        assert L.hl_route_gather(h.ptr, S, *args, None) == 1, args
        assert L.hl_route_gather_bwd(h.ptr, S, args[0], args[1], args[4], args[5], args[2], args[3], None) == 1, args
        assert L.hl_route_combine(h.ptr, S, args[0], args[1], args[4], args[5], None, args[2], args[3], None) == 1, args
        assert L.hl_route_combine_bwd(h.ptr, S, args[0], args[1], args[2], args[3], None, 0, None, args[4], args[5], None,
                                      None) == 1, args
    assert L.hl_route_combine_bwd(h.ptr, S, 0, 8, X, 8, None, 8, None, R, 8, X, None) == 1  # dweights without rows
    # more than one tile of assignments needs a workspace, of the size it asks for
    big = ids(0, 9000, 1, 3)
    q = Plan(h, big, 3)
    assert status(hl.hl_route_plan, h, q.route, q.experts, None) == 1
    assert status(hl.hl_route_plan, h, q.route, q.experts, q.ws[:8]) == 3
    assert hl.hl_last_device_error(h) == 0


def test_stream_and_graphs(h):
    """On another stream than the tensors' own, and captured: two graphs that share a workspace, replayed in turn with
    eager calls between them, each replay equal to the eager result."""
    cases = []
    for t, k, E, dim in ((20000, 2, 16, 96), (9000, 3, 40, 64)):
        cases.append([t, k, E, dim, ids(t, t, k, E, 0.1), torch.randn(t, dim, device="cuda"),
                      torch.rand(t, k, device="cuda")])
    ws = torch.zeros(max(hl.hl_route_workspace_bytes(c[0], c[1], c[2]) for c in cases), dtype=torch.uint8, device="cuda")
    made = []
    for t, k, E, dim, e, x, w in cases:
        p = Plan(h, e, E, capacity=2 * t * k // E, align=8)
        rows, out = torch.zeros(p.n_rows, dim, device="cuda"), torch.zeros(t, dim, device="cuda")
        drows, dw, dx = torch.zeros_like(rows), torch.zeros_like(w), torch.zeros_like(x)

        def step(p=p, x=x, w=w, rows=rows, out=out, drows=drows, dw=dw, dx=dx):
            hl.hl_route_plan(h, p.route, p.experts, ws)
            hl.hl_route_gather(h, p.route, x, rows)
            hl.hl_route_combine(h, p.route, rows, w, out)
            hl.hl_route_combine_bwd(h, p.route, out, rows, w, drows, dw)
            hl.hl_route_gather_bwd(h, p.route, drows, dx)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        made.append((g, step, p, x, w, [p.pos, p.order, rows, out, drows, dw, dx]))
    for turn in range(4):
        for g, step, p, x, w, outs in made:
            gen = torch.Generator(device="cuda").manual_seed(turn)
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            p.experts.copy_(ids(turn, *p.experts.shape, p.args[0], 0.2).cuda())
            step()
            torch.cuda.synchronize()
            want = [o.clone() for o in outs]
            used = int(p.offsets[-1])
            for o in outs:
                o.zero_()
            g.replay()
            torch.cuda.synchronize()
            for i, (o, v) in enumerate(zip(outs, want)):
                n = used if i in (1, 2, 4) else o.shape[0]  # (order, rows, drows: the rows in use)
                assert torch.equal(o[:n], v[:n]), (turn, i)
    assert hl.hl_last_device_error(h) == 0
