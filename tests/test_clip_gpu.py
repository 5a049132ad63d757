"""The global gradient norm and clipping on the GPU: lists of dense tensors and
the tables' coalesced gradient against sums in 64 bits, and the clipped table
update bit for bit against the unclipped one with the scaled learning rate."""
import math

import numpy as np
import pytest
import torch

from paper_2204_05436_amd import configs, hotline as hl, workload as W
from paper_2204_05436_amd.runner import HotPath, to_device
from parity_lib import make_table

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24  # half a step of fp32, relative


@pytest.fixture(scope="module")
def h():
    x = hl.hl_create([1], 1, "f32", 1)
    yield x
    x.close()


@pytest.fixture(scope="module")
def ws():
    return torch.zeros(hl.hl_grad_workspace_bytes(), dtype=torch.uint8, device="cuda")


def make(sizes, dtypes, seed, shift=0, scale=1.0):
    """Tensors of those sizes packed back to back by type, the first `shift` elements into its buffer."""
    g, bufs, at = torch.Generator(device="cuda").manual_seed(seed), {}, []
    for i, n in enumerate(sizes):
        d = dtypes[i % len(dtypes)]
        at.append((d, bufs.get(d, shift), n))
        bufs[d] = bufs.get(d, shift) + n
    bufs = {d: (torch.randn(n + 9, generator=g, device="cuda") * scale).to(DT[d]) for d, n in bufs.items()}
    return [bufs[d][o:o + n] for d, o, n in at], bufs


def norm_of(ts):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in ts))


def coef(norm, max_norm):
    return 0.0 if not math.isfinite(norm) else (1.0 if norm <= max_norm else max_norm / norm)


def clipped_ok(src, dst, c):
    f = torch.finfo(src.dtype)
    ref = src.double() * c
    # c and the product are each rounded to fp32 (U each), the product to the type (half a step)
    tol = ref.abs() * ((1 + U) ** 2 * (1 + f.eps / 2) - 1) + f.smallest_normal * f.eps / 2
    return bool(((dst.double() - ref).abs() <= tol).all())


def sq_ok(got, want):
    # squares of 24-bit values are exact in fp64; a chain of at most 2^13 additions of positive terms
    return abs(got - want) <= 2.0 ** -39 * want


LISTS = [([0], ["f32"]), ([1], ["bf16"]), ([0, 5, 0, 7, 0], ["f32"]), ([8191, 8192, 8193, 16385], ["f32"]),
         ([16383, 16384, 16385, 1], ["bf16", "f16"]), ([3] * 111 + [4] * 3, ["f32", "bf16", "f16"]),
         ([100_003, 1, 0, 65_537] * 60, ["bf16", "f32"]), ([40_000_011], ["f16"]), ([70_000_001, 3], ["f32", "bf16"])]


@pytest.mark.parametrize("sizes,dtypes", LISTS, ids=lambda v: str(len(v)) if isinstance(v[0], int) else "-".join(v))
@pytest.mark.parametrize("shift", [0, 1])
def test_dense(h, ws, sizes, dtypes, shift):
    ts, bufs = make(sizes, dtypes, len(sizes) + sum(sizes) % 97, shift)
    sq, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    grads = hl.GradList(ts)
    hl.hl_grad_sq(h, grads, sq, ws)
    want = norm_of(ts)
    assert sq_ok(float(sq), want * want)
    again = torch.zeros_like(sq)
    hl.hl_grad_sq(h, grads, again, ws)
    assert torch.equal(sq, again)
    out, obufs = make(sizes, dtypes, 1, shift)  # (other addresses, other contents)
    keep = {d: b.clone() for d, b in obufs.items()}
    for max_norm in (want * 2, want / 3):
        c = coef(want, max_norm)
        hl.hl_grad_clip(h, hl.GradList(ts, out), sq, max_norm, norm)
        assert abs(float(norm) - want) <= 2 * U * want
        for s, d in zip(ts, out):
            assert clipped_ok(s, d, c)
        for d, b in obufs.items():  # nothing outside the tensors
            n = sum(t.numel() for t in out if t.dtype == b.dtype)
            assert torch.equal(b[:shift], keep[d][:shift]) and torch.equal(b[shift + n:], keep[d][shift + n:])
    hl.hl_grad_clip(h, grads, sq, want / 3)  # in place: the same values
    for s, d in zip(ts, out):
        assert torch.equal(s, d)
    hl.hl_grad_sq(h, grads, sq, ws)
    hl.hl_grad_clip(h, grads, sq, want, norm)  # (now below the bound: nothing changes)
    for s, d in zip(ts, out):
        assert torch.equal(s, d)
    assert hl.hl_last_device_error(h) == 0


def test_long_tensor(h, ws):
    """A tensor of more elements than one entry of a launch takes (2^29), at an odd address."""
    n = (1 << 29) + 12_345
    buf = torch.full((n + 2,), 0.5, dtype=torch.bfloat16, device="cuda")
    t = buf[1:-1]
    t[-1] = 3.0
    t[(1 << 29) - 1] = -2.0
    sq = torch.zeros(1, dtype=torch.float64, device="cuda")
    hl.hl_grad_sq(h, hl.GradList([t]), sq, ws)
    assert float(sq) == 0.25 * (n - 2) + 9 + 4  # (a multiple of 1/4 below 2^53)
    norm = math.sqrt(float(sq))
    hl.hl_grad_clip(h, hl.GradList([t]), sq, float(np.float32(norm / 4)))
    c = float(np.float32(norm / 4)) / norm
    for at, v in ((0, 0.5), ((1 << 29) - 1, -2.0), (1 << 29, 0.5), (n - 2, 0.5), (n - 1, 3.0)):
        assert clipped_ok(torch.tensor([v], dtype=torch.bfloat16, device="cuda"), t[at:at + 1], c)
    assert int((t == t[0]).sum()) == n - 2 and float(buf[0]) == 0.5 and float(buf[-1]) == 0.5


def test_many_launches(h, ws):
    """More tensors than the sums of eight launches' blocks have room for: added up in between."""
    m, n = 2300, 150_001
    flat = torch.ones(m * n, device="cuda")
    flat[:n] = 2.0
    flat[-n:] = 3.0
    ts = [flat[i * n:(i + 1) * n] for i in range(m)]
    sq, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    grads = hl.GradList(ts)
    for _ in range(2):
        hl.hl_grad_sq(h, grads, sq, ws)
        want = float(n) * (m - 2 + 4 + 9)
        assert float(sq) == want
    hl.hl_grad_clip(h, grads, sq, float(np.float32(math.sqrt(want) / 8)), norm)
    assert abs(float(norm) - math.sqrt(want)) <= 2 * U * float(norm)
    c = float(np.float32(math.sqrt(want) / 8)) / math.sqrt(want)
    for i, v in ((0, 2.0), (1, 1.0), (m // 2, 1.0), (m - 1, 3.0)):
        assert clipped_ok(torch.full((n,), v, device="cuda"), ts[i], c)
    assert torch.equal(flat[n:-n], flat[n].expand(flat.numel() - 2 * n))
    assert hl.hl_last_device_error(h) == 0


def test_empty_list(h, ws):
    sq, norm = torch.full((1,), 7.0, dtype=torch.float64, device="cuda"), torch.full((1,), 7.0, device="cuda")
    hl.hl_grad_sq(h, hl.GradList([]), sq, ws)
    assert float(sq) == 0
    hl.hl_grad_clip(h, hl.GradList([]), sq, 1.0, norm)
    assert float(norm) == 0


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_not_finite(h, ws, dt, value):
    """A gradient that is not finite: the norm says so, and every clipped value is zero."""
    ts, _ = make([1000, 30], [dt], 4)
    ts[0][777] = value
    sq, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    hl.hl_grad_sq(h, hl.GradList(ts), sq, ws)
    out = [torch.full_like(t, 5.0) for t in ts]
    for max_norm in (1.0, float("inf")):
        hl.hl_grad_clip(h, hl.GradList(ts, out), sq, max_norm, norm)
        assert (math.isnan(float(norm)) if math.isnan(value) else float(norm) == math.inf)
        assert all(not bool(o.any()) for o in out)
    hl.hl_grad_clip(h, hl.GradList(ts), sq, 1.0)
    assert all(not bool(t.any()) for t in ts)


@pytest.mark.parametrize("dt", DT)
def test_extremes(h, ws, dt):
    """The largest and smallest values of a type: squares past fp32's range are counted, and clipping brings them
    down; a bound of zero gives zeros, an infinite one changes nothing."""
    f = torch.finfo(DT[dt])
    sq, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    for v in (f.max, f.smallest_normal, f.smallest_normal * f.eps):
        t = torch.full((333,), v, dtype=DT[dt], device="cuda")
        want = float(t[0].double()) * math.sqrt(333)
        hl.hl_grad_sq(h, hl.GradList([t]), sq, ws)
        assert sq_ok(float(sq), want * want)
        for max_norm in (want / 2, 0.0, math.inf, 1.0, 1e-6, 1e-30):
            m = math.inf if max_norm > 3e38 else float(np.float32(max_norm))
            out = torch.empty_like(t)
            hl.hl_grad_clip(h, hl.GradList([t], [out]), sq, m, norm)
            assert clipped_ok(t, out, coef(want, m))


def test_several_parts(h, ws):
    """A norm of parts: their order in sq is the order of the sum, and more than 64 of them are taken too."""
    t = torch.randn(1000, device="cuda")
    norm = torch.zeros(1, device="cuda")
    for n in (1, 2, 64, 65, 1000):
        sq = torch.rand(n, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
        want = math.sqrt(float(sq.sum()))
        out = torch.empty_like(t)
        hl.hl_grad_clip(h, hl.GradList([t], [out]), sq, want / 4, norm)
        assert abs(float(norm) - want) <= 2 * U * want
        assert clipped_ok(t, out, float(np.float32(want / 4)) / want)


def test_dense_refusals(h, ws):
    L, t = hl.lib(), torch.zeros(64, device="cuda")
    sq = torch.zeros(1, dtype=torch.float64, device="cuda")
    W, S, n = ws.data_ptr(), sq.data_ptr(), ws.numel()

    def entry(src=t.data_ptr(), dst=t.data_ptr(), size=64, dtype=0):
        return (hl.GradStruct * 1)(hl.GradStruct(src, dst, size, dtype))

    assert L.hl_grad_sq(h.ptr, entry(), -1, S, W, n, None) == 1
    assert L.hl_grad_sq(h.ptr, None, 1, S, W, n, None) == 1
    for bad in [entry(src=None), entry(src=t.data_ptr() + 2), entry(size=-1), entry(dtype=3), entry(dtype=-1)]:
        assert L.hl_grad_sq(h.ptr, bad, 1, S, W, n, None) == 1
        assert L.hl_grad_clip(h.ptr, bad, 1, S, 1, 1.0, None, None) == 1
    for bad in [entry(dst=None), entry(dst=t.data_ptr() + 2), entry(dst=t.data_ptr() + 16), entry(dst=t.data_ptr() - 4)]:
        assert L.hl_grad_clip(h.ptr, bad, 1, S, 1, 1.0, None, None) == 1
    assert L.hl_grad_sq(h.ptr, entry(size=(1 << 40) + 1), 1, S, W, n, None) == 5
    assert L.hl_grad_sq(h.ptr, entry(), 1, None, W, n, None) == 1
    assert L.hl_grad_sq(h.ptr, entry(), 1, S + 4, W, n, None) == 1
    assert L.hl_grad_sq(h.ptr, entry(), 1, S, None, n, None) == 1
    assert L.hl_grad_sq(h.ptr, entry(), 1, S, W, n // 2, None) == 3
    assert L.hl_grad_clip(h.ptr, entry(), 1, None, 1, 1.0, None, None) == 1
    assert L.hl_grad_clip(h.ptr, entry(), 1, S, 0, 1.0, None, None) == 1
    for m in (-1.0, float("nan")):
        assert L.hl_grad_clip(h.ptr, entry(), 1, S, 1, m, None, None) == 1
    assert L.hl_grad_clip(h.ptr, entry(), 1, S, 1, 1.0, S + 2, None) == 1
    assert hl.hl_last_device_error(h) == 0


# ------------------------------------------------------------------ the tables
class Tables:
    """A mini-batch over tables whose first rows are hot; staging holds the cold rows in use."""

    def __init__(self, tables, rows, dim, dt, B, bag=0.0, seed=0, hot=0.3, alpha=1.2, invalid=0.0):
        g = np.random.RandomState(seed)
        self.B, self.T, self.dim, self.dt = B, tables, dim, dt
        self.rows = [max(2, rows // (i + 1)) for i in range(tables)]
        nh = [max(1, int(r * hot)) for r in self.rows]
        self.n_hot, n_bags = sum(nh), B * tables
        lens = np.ones(n_bags, np.int64) if not bag else g.poisson(bag, n_bags)
        self.ptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.bag = np.repeat(np.arange(n_bags), lens)
        t = self.bag % tables
        r = (g.zipf(alpha, self.bag.size) - 1) % np.array(self.rows)[t]
        first, first_hot = np.cumsum(self.rows) - self.rows, np.cumsum(nh) - nh
        cold = r >= np.array(nh)[t]
        ids, inv = np.unique(np.where(cold, first[t] + r, -1), return_inverse=True)
        skip = int(ids.size and ids[0] == -1)
        self.n_stg, self.L = max(1, ids.size - skip), self.bag.size
        self.row = np.where(cold, self.n_hot + inv - skip, first_hot[t] + r)
        self.h = hl.hl_create(self.rows, dim, dt, self.n_hot)
        ids = np.concatenate([np.arange(f, f + n) for f, n in zip(first, nh)]).astype(np.int32)
        hl.hl_set_hot(self.h, torch.from_numpy(ids).cuda(), self.n_hot)
        codes = self.row.astype(np.int32)
        self.codes, self.ptr_d = torch.from_numpy(codes).cuda(), torch.from_numpy(self.ptr).cuda()
        w = torch.randn(self.n_hot + self.n_stg, dim, generator=torch.Generator().manual_seed(seed)) * 0.1
        self.w = w.to(DT[dt]).cuda()
        self.dY = torch.randn(n_bags, dim, generator=torch.Generator().manual_seed(seed + 1)).cuda()
        self.ws = torch.zeros(hl.hl_workspace_bytes(self.h, self.L, n_bags, B), dtype=torch.uint8, device="cuda")
        self.sq = torch.zeros(1, dtype=torch.float64, device="cuda")
        self.norm = torch.zeros(1, device="cuda")

    def shape(self):
        return self.n_stg, self.B, self.T, self.L

    def plan(self, ids=None):
        hl.hl_embbag_bwd_plan(self.h, self.n_stg, self.codes, self.ptr_d, self.B, self.T, self.L, ids, None,
                              self.B if ids is None else ids.numel(), self.ws)

    def norm_(self, dY=None, sq=None, **kw):
        hl.hl_embbag_bwd_norm(self.h, *self.shape(), self.dY if dY is None else dY, self.sq if sq is None else sq, self.ws, **kw)

    def clip(self, w, max_norm, lr, sq=None, **kw):
        hl.hl_embbag_bwd_clip(self.h, w[:self.n_hot], w[self.n_hot:], *self.shape()[:1], self.B, self.T, self.L,
                              self.sq if sq is None else sq, max_norm, lr, self.ws, self.norm, **kw)

    def apply(self, w, lr):
        hl.hl_embbag_bwd_apply(self.h, w[:self.n_hot], w[self.n_hot:], *self.shape(), self.dY, lr, self.ws)

    def sums(self, samples=None):
        """The coalesced gradient, and the sum of its terms' sizes and their number, in 64 bits."""
        take = np.ones(self.L, bool) if samples is None else np.isin(self.bag // self.T, samples)
        row, bag = torch.from_numpy(self.row[take]).cuda(), torch.from_numpy(self.bag[take]).cuda()
        G = torch.zeros(self.w.shape, dtype=torch.float64, device="cuda")
        A, n = G.clone(), torch.zeros(self.w.shape[0], dtype=torch.float64, device="cuda")
        d = self.dY.double()[bag]
        return (G.index_add_(0, row, d), A.index_add_(0, row, d.abs()),
                n.index_add_(0, row, torch.ones(row.numel(), dtype=torch.float64, device="cuda")))


CASES = [(1, 50, 1, "f32", 1, 0.0), (8, 5000, 16, "f32", 300, 0.0), (26, 3000, 64, "f32", 700, 0.0),
         (3, 40, 64, "f32", 3000, 0.0), (5, 2000, 20, "f32", 257, 3.0), (4, 900, 128, "bf16", 300, 18.0),
         (2, 10, 96, "bf16", 2000, 0.0), (3, 500, 7, "f32", 333, 2.0), (2, 300, 130, "bf16", 150, 4.0),
         (1, 3, 32, "f32", 9000, 0.0), (2, 700, 10, "bf16", 500, 1.5), (1, 100, 520, "f32", 200, 2.0),
         (2, 100, 520, "bf16", 200, 2.0), (6, 200, 8, "f32", 64, 0.0), (70, 30, 4, "f32", 90, 0.0)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_tables(case):
    t = Tables(*case, seed=case[1])
    try:
        G, A, n = t.sums()
        # an fp32 sum of n terms is off by (n - 1) U of their sizes at most; bags add nothing (one row of dY each)
        off = n[:, None] * U * A
        want, slack = float(G.square().sum()), float((2 * G.abs() * off + off * off).sum())
        lr = 0.25
        for how in ("plan", "fwd_plan"):
            if how == "plan":
                t.plan()
            else:
                out = torch.zeros_like(t.dY)
                hl.hl_embbag_fwd_plan(t.h, t.w[:t.n_hot], t.w[t.n_hot:], t.n_stg, t.codes, t.ptr_d, t.B, t.T, t.L,
                                      out, t.ws)
            t.norm_()
            assert abs(float(t.sq) - want) <= slack + 2.0 ** -39 * want
            # no clipping: bit for bit the plain update
            a, b = t.w.clone(), t.w.clone()
            t.clip(a, math.inf, lr)
            assert abs(float(t.norm) - math.sqrt(float(t.sq))) <= 2 * U * float(t.norm)
            t.apply(b, lr)
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
            # clipping: bit for bit the plain update with the scaled learning rate
            m = float(np.float32(math.sqrt(want) / 7))
            c = np.float32(m / math.sqrt(float(t.sq)))
            a, b = t.w.clone(), t.w.clone()
            t.clip(a, m, lr)
            t.apply(b, float(np.float32(lr) * c))
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
            ref = t.w.double() - lr * float(c) * G
            f = torch.finfo(t.w.dtype)
            # the sum, the two scalings and the subtraction in fp32, the row's rounding
            upd = lr * float(c) * (G.abs() + off)
            tol = lr * float(c) * off + 4 * U * (upd + t.w.double().abs()) + f.eps / 2 * ref.abs() * (1 + 2 * U)
            assert ((a.double() - ref).abs() <= tol * (1 + f.eps)).all()
            # a bound of zero, and a norm that is not finite: no row changes
            a = t.w.clone()
            t.clip(a, 0.0, lr)
            t.clip(a, 1.0, lr, sq=torch.tensor([float(t.sq), math.inf], dtype=torch.float64, device="cuda"))
            assert math.isinf(float(t.norm))
            t.clip(a, 1.0, lr, sq=torch.tensor([math.nan], dtype=torch.float64, device="cuda"))
            assert math.isnan(float(t.norm)) and torch.equal(a, t.w)
            # a second step with the same sums
            a, b = t.w.clone(), t.w.clone()
            for _ in range(2):
                t.clip(a, math.inf, lr)
                t.apply(b, lr)
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()


@pytest.mark.parametrize("dt,dim", [("f32", 64), ("bf16", 40), ("f32", 3)])
def test_tables_selected_samples(dt, dim):
    """A plan over some samples: only their lookups count, other rows stay."""
    t = Tables(4, 300, dim, dt, 200, 2.5, seed=3)
    try:
        ids = np.arange(1, 200, 3, dtype=np.int32)
        t.plan(torch.from_numpy(ids).cuda())
        t.norm_()
        G, A, n = t.sums(ids)
        off = n[:, None] * U * A
        want, slack = float(G.square().sum()), float((2 * G.abs() * off + off * off).sum())
        assert abs(float(t.sq) - want) <= slack + 2.0 ** -39 * want
        a, b = t.w.clone(), t.w.clone()
        t.clip(a, math.inf, 0.5)
        t.apply(b, 0.5)
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(a[n == 0], t.w[n == 0])
    finally:
        t.h.close()


def test_tables_gradient_by_differences():
    """The clipped step against differences of the pooled sum's dot product with dY: f = <dY, pool(w)> is linear in w,
    so the step is -lr c times its differences."""
    t = Tables(2, 6, 3, "f32", 5, 1.5, seed=9)
    try:
        t.w = torch.round(t.w * 4096) / 4096
        t.dY = torch.round(t.dY * 64) / 64
        out = torch.zeros_like(t.dY)

        def f(w):
            hl.hl_embbag_fwd(t.h, w[:t.n_hot], w[t.n_hot:], t.n_stg, t.codes, t.ptr_d, t.B, t.T, t.L, None, None, t.B, out)
            return float((out.double() * t.dY.double()).sum())

        t.plan()
        t.norm_()
        a = t.w.clone()
        t.clip(a, 1.0, 1.0)
        c = 1.0 / math.sqrt(float(t.sq))
        assert c < 1
        for i in range(t.w.numel()):
            lo, hi = t.w.clone(), t.w.clone()
            lo.view(-1)[i] -= 0.125
            hi.view(-1)[i] += 0.125
            g = (f(hi) - f(lo)) / 0.25  # (exact: every value is a small multiple of 2^-12)
            w = float(t.w.view(-1)[i])
            assert abs(float(a.view(-1)[i]) - (w - c * g)) <= 4 * U * (abs(w) + abs(c * g)) + 1e-12
    finally:
        t.h.close()


def test_tables_many_lookups():
    """More lookups than one dimension of the clipped update's grid takes (2^26), of few rows and of many."""
    L, bags, n_hot, n_stg = (1 << 26) + 4_000_003, 1000, 30_000_000, 5
    h = hl.hl_create([n_hot + 100], 1, "f32", n_hot)
    try:
        hl.hl_set_hot(h, torch.arange(n_hot, dtype=torch.int32, device="cuda"), n_hot)
        g = torch.Generator(device="cuda").manual_seed(1)
        codes = torch.randint(0, n_hot + n_stg, (L,), dtype=torch.int32, device="cuda", generator=g)
        codes[: L // 4] %= 100  # (long runs)
        ptr = torch.linspace(0, L, bags + 1, dtype=torch.float64, device="cuda").to(torch.int32)
        dY = torch.randint(-4, 5, (bags, 1), device="cuda", generator=g).float()
        ws = torch.zeros(hl.hl_workspace_bytes(h, L, bags, bags), dtype=torch.uint8, device="cuda")
        sq = torch.zeros(1, dtype=torch.float64, device="cuda")
        a = torch.randn(n_hot + n_stg, 1, device="cuda", generator=g)
        b = a.clone()
        shape = (n_stg, bags, 1, L)
        hl.hl_embbag_bwd_plan(h, n_stg, codes, ptr, bags, 1, L, None, None, bags, ws)
        hl.hl_embbag_bwd_norm(h, *shape, dY, sq, ws)
        bag = torch.repeat_interleave(torch.arange(bags, device="cuda"), (ptr[1:] - ptr[:-1]).long())
        G = torch.zeros(n_hot + n_stg, dtype=torch.float64, device="cuda").index_add_(0, codes, dY.double()[bag, 0])
        assert float(G.abs().max()) < 2 ** 24  # (whole numbers: exact sums)
        assert sq_ok(float(sq), float(G.square().sum()))
        hl.hl_embbag_bwd_clip(h, a[:n_hot], a[n_hot:], *shape, sq, math.inf, 0.5, ws)
        hl.hl_embbag_bwd_apply(h, b[:n_hot], b[n_hot:], *shape, dY, 0.5, ws)
        assert torch.equal(a, b)
        assert hl.hl_last_device_error(h) == 0
    finally:
        h.close()


def test_tables_unaligned_rows():
    """Rows and gradients at addresses that allow narrower loads only."""
    t = Tables(3, 400, 64, "f32", 150, 2.0, seed=5)
    try:
        G, A, n = t.sums()
        buf, dbuf = torch.zeros(t.w.numel() + 1, device="cuda"), torch.zeros(t.dY.numel() + 2, device="cuda")
        w, d = buf[1:].view_as(t.w), dbuf[2:].view_as(t.dY)
        d.copy_(t.dY)
        for dY in (t.dY, d):
            w.copy_(t.w)
            t.plan()
            t.norm_(dY)
            t.clip(w, math.inf, 0.5)
            tol = 0.5 * n[:, None] * U * A + 4 * U * (G.abs() + t.w.double().abs())
            assert ((w.double() - (t.w.double() - 0.5 * G)).abs() <= tol).all()
    finally:
        t.h.close()


def test_tables_refusals():
    t = Tables(3, 100, 16, "f32", 40, 2.0, seed=1)
    try:
        def refused(f, want=1):
            with pytest.raises(hl.HotlineError) as e:
                f()
            assert e.value.status == want

        w = t.w.clone()
        refused(t.norm_)                              # no plan
        t.plan()
        refused(lambda: t.clip(w, 1.0, 0.1))          # no norm
        refused(lambda: t.norm_(dY=0))
        t.norm_()
        refused(lambda: t.clip(w, -1.0, 0.1))
        refused(lambda: t.clip(w, math.nan, 0.1))
        S = t.sq.data_ptr()
        L = hl.lib()
        args = (t.n_stg, t.B, t.T, t.L)
        wh, st, W, nb = w.data_ptr(), w[t.n_hot:].data_ptr(), t.ws.data_ptr(), t.ws.numel()
        assert L.hl_embbag_bwd_norm(t.h.ptr, *args, t.dY.data_ptr(), None, W, nb, None) == 1
        assert L.hl_embbag_bwd_norm(t.h.ptr, *args, t.dY.data_ptr(), S + 4, W, nb, None) == 1
        assert L.hl_embbag_bwd_norm(t.h.ptr, *args, t.dY.data_ptr(), S, W, 4096, None) == 3
        assert L.hl_embbag_bwd_norm(t.h.ptr, t.n_stg + 1, *args[1:], t.dY.data_ptr(), S, W, nb, None) == 1
        for a in [(None, st, S, 1), (wh, None, S, 1), (wh, st, None, 1), (wh, st, S + 4, 1), (wh, st, S, 0)]:
            assert L.hl_embbag_bwd_clip(t.h.ptr, a[0], a[1], *args, a[2], a[3], 1.0, 0.1, W, nb, None, None) == 1
        assert L.hl_embbag_bwd_clip(t.h.ptr, wh, st, *args, S, 1, 1.0, 0.1, W, nb, S + 2, None) == 1
        # the second half of the split update does not take the norm's sums, nor the clipped one the split's
        assert L.hl_embbag_bwd_apply_part(t.h.ptr, wh, st, *args, t.dY.data_ptr(), 0.1, 2, W, nb, None) == 1
        hl.hl_embbag_bwd_apply_part(t.h, w[:t.n_hot], w[t.n_hot:], *args, t.dY, 0.1, 1, t.ws)
        refused(lambda: t.clip(w, 1.0, 0.1))
        t.plan()
        t.norm_()
        t.plan()
        refused(lambda: t.clip(w, 1.0, 0.1))          # another call in between
        t.norm_()
        hl.hl_set_hot(t.h, torch.arange(3, dtype=torch.int32, device="cuda"), 3)
        refused(lambda: t.clip(w, 1.0, 0.1))          # another hot set
        assert hl.hl_last_device_error(t.h) == 0
    finally:
        t.h.close()


def test_tables_empty():
    """No lookups at all: a norm of zero, no rows written."""
    h = hl.hl_create([10], 8, "f32", 4)
    try:
        hl.hl_set_hot(h, torch.arange(4, dtype=torch.int32, device="cuda"), 4)
        ptr = torch.zeros(4, dtype=torch.int32, device="cuda")
        ws = torch.zeros(hl.hl_workspace_bytes(h, 0, 3, 3), dtype=torch.uint8, device="cuda")
        sq, norm = torch.full((1,), 3.0, dtype=torch.float64, device="cuda"), torch.full((1,), 3.0, device="cuda")
        w, codes = torch.ones(4, 8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        hl.hl_embbag_bwd_plan(h, 0, codes, ptr, 3, 1, 0, None, None, 3, ws)
        hl.hl_embbag_bwd_norm(h, 0, 3, 1, 0, torch.zeros(3, 8, device="cuda"), sq, ws)
        assert float(sq) == 0
        hl.hl_embbag_bwd_clip(h, w, None, 0, 3, 1, 0, sq, 1.0, 0.1, ws, norm)
        assert float(norm) == 0 and bool((w == 1).all())
        assert hl.hl_last_device_error(h) == 0
    finally:
        h.close()


@pytest.mark.parametrize("name", ["tiny", "multi-hot"])
def test_path_step(name):
    """The path's step with a bound on the norm: far above it bit for bit the plain step, below it the plain step with
    the scaled learning rate; a dense part counts in the norm."""
    w = configs.scaled(configs.WORKLOADS[name], batch=200, row_scale=0.02, name=name + "-clip")
    rows = W.table_rows(w)
    prof = [W.make_batch(w, rows, i) for i in range(3)]
    mb = W.make_batch(w, rows, 3)
    table = make_table(w, int(rows.sum(dtype=np.int64)))
    hp = HotPath(w, rows, table, max(x.n_lookups for x in prof + [mb]), w.batch)
    try:
        hp.learn([to_device(p, "cuda") for p in prof])
        b = to_device(mb, "cuda", W.make_dy(w, 3, mb.n_bags))
        start = hp.w_hot.clone()

        def step(**kw):
            hp.w_hot.copy_(start)
            hp.step(b, mode="sequential", **kw)
            return hp.w_hot.clone(), hp.staging[:int(hp.n_cold.item())].clone()

        same = lambda x, y: all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(x, y))
        for split in (True, False):
            assert same(step(split_fwd=split, max_norm=math.inf), step(split_fwd=split))
            norm = math.sqrt(float(hp.norm_parts))
            assert abs(float(hp.grad_norm) - norm) <= 2 * U * norm
            m = float(np.float32(norm / 5))
            parts = torch.tensor([0.0, 3 * norm * norm], dtype=torch.float64, device="cuda")  # (the norm is twice this)
            for p, full in ((None, norm), (parts, None)):
                got = step(split_fwd=split, max_norm=m, norm_parts=p)
                if p is not None:
                    full = math.sqrt(float(parts[0]) + float(parts[1]))
                    assert abs(full - 2 * norm) <= 1e-9 * norm
                lr = float(np.float32(w.lr) * np.float32(m / full))
                assert same(got, step(split_fwd=split, lr=lr))
                assert not same(got, step(split_fwd=split))
        for kw in (dict(mode="pipelined"), dict(mode="fwdbwd")):
            with pytest.raises(ValueError):
                hp.step(b, max_norm=1.0, **kw)
        with pytest.raises(ValueError):
            hp.step(b, mode="sequential", norm_parts=parts)
        assert hp.device_error() == 0
    finally:
        hp.close()
        table.close()


def test_stream_and_graphs(h, ws):
    """Dense and table gradients clipped by one norm, on another stream and captured: two graphs sharing a workspace,
    replayed in turn with eager calls between them, each replay equal to the eager result."""
    tabs = [Tables(4, 900, 32, "f32", 250, 2.0, seed=1), Tables(8, 2000, 64, "bf16", 500, 0.0, seed=2)]
    made = []
    try:
        for i, t in enumerate(tabs):
            ts, _ = make([70_001, 5, 40_000], ["f32", "bf16"], i)
            out = [torch.empty_like(x) for x in ts]
            sq, norm = torch.zeros(2, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
            w = t.w.clone()

            def step(t=t, grads=hl.GradList(ts, out), sq=sq, norm=norm, w=w):
                t.plan()
                t.norm_(sq=sq[1:])
                hl.hl_grad_sq(h, grads, sq, ws)
                hl.hl_grad_clip(h, grads, sq, 10.0, norm)
                t.clip(w, 10.0, 0.1, sq=sq)

            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            made.append((g, step, t, ts, out + [sq, norm, w]))
        for turn in range(4):
            for g, step, t, ts, outs in made:
                for x in ts + [t.dY]:
                    x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(turn)) * (turn + 0.5))
                w = outs[-1]
                w.copy_(t.w)
                step()
                torch.cuda.synchronize()
                want = [o.clone() for o in outs]
                full = math.sqrt(norm_of(ts) ** 2 + float(want[-3][1]))
                assert abs(float(want[-2]) - full) <= 2 * U * full
                for o in outs:
                    o.zero_()
                w.copy_(t.w)
                g.replay()
                torch.cuda.synchronize()
                for o, v in zip(outs, want):
                    assert torch.equal(o, v)
                assert hl.hl_last_device_error(t.h) == 0
        assert hl.hl_last_device_error(h) == 0
    finally:
        for t in tabs:
            t.h.close()
