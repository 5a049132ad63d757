"""Timed cases of routing to experts and of gradient clipping, the operators that stand around the embedding
tables in a training or serving program, each through the library's public entry points.

Kinds of case:

  dispatch     tokens sorted by expert and copied into the experts' blocks (hl_route_plan, hl_route_gather)
  combine      the experts' rows back at their tokens, weighted and summed (hl_route_combine)
  experts_bwd  the gradients of both (hl_route_combine_bwd, hl_route_gather_bwd)
  clip         the global norm of many gradient tensors, and the clipped tensors (hl_grad_sq, hl_grad_clip)
  tables       the coalesced gradient of a mini-batch's lookups, its norm, and the clipped SGD update of the
               rows (hl_embbag_bwd_plan, hl_embbag_bwd_norm, hl_embbag_bwd_clip)

A token's experts are k different ones, drawn with popularity that falls off over the experts; a share `drop` of
the tokens is padding (no expert), and `capacity` (a factor of the mean load) drops what is past it.  The lookups of
a table follow a power law over its rows, the first `hot` share of which lies in the hot cache."""
from __future__ import annotations

import math
import sys

import numpy as np
import torch

own = False
LR = 0.5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _route(name, op, tokens, k, experts, dim, dtype, drop=0.0, capacity=0.0, align=1, slack=0):
    return dict(name=name, op=op, tokens=tokens, k=k, experts=experts, dim=dim, dtype=dtype, drop=drop,
                capacity=capacity, align=align, slack=slack)


def _clip(name, tensors, total, dtypes, packed, max_norm=1.0):
    return dict(name=name, op="clip", tensors=tensors, total=total, dtypes=dtypes, packed=packed, max_norm=max_norm)


def _tables(name, tables, rows, dim, dtype, batch, hot, bag=0.0, alpha=1.1, max_norm=1.0):
    return dict(name=name, op="tables", tables=tables, rows_lo=rows[0], rows_hi=rows[1], dim=dim, dtype=dtype,
                batch=batch, hot=hot, bag=bag, alpha=alpha, max_norm=max_norm)


def listed():
    return [
        # one token served: launches and latency
        _route("dispatch-one", "dispatch", 1, 2, 8, 1024, "bf16"),
        # a training batch, fine-grained experts whose products run over tiles of 16 rows
        _route("dispatch-batch", "dispatch", 4096, 8, 64, 2048, "bf16", align=16),
        # a padded batch with a capacity, rows of an odd length
        _route("dispatch-ragged", "dispatch", 10007, 3, 37, 333, "f32", drop=0.1, capacity=1.1),
        # one decoding step of a few dozen sequences
        _route("combine-few", "combine", 48, 8, 128, 4096, "bf16"),
        # long prompts, wide rows
        _route("combine-large", "combine", 16384, 4, 32, 4096, "f16"),
        # a training batch's gradients, few wide experts
        _route("experts-bwd-wide", "experts_bwd", 8192, 2, 8, 4096, "bf16", align=16),
        # gradients in f32 at sizes that divide nothing, rows padded to a stride
        _route("experts-bwd-ragged", "experts_bwd", 2999, 6, 60, 769, "f32", drop=0.1, capacity=1.0, slack=7),
        # the dense part of a click model: a few small layers
        _clip("clip-small", 12, 600_000, "f32", False),
        # the gradients of a large model's layers
        _clip("clip-layers", 290, 400_000_000, "bf16", False),
        # many tensors of several types packed back to back, at any alignment
        _clip("clip-mixed", 701, 40_000_000, "f32,bf16,f16", True),
        # the one-hot click model
        _tables("tables-large", 26, (100, 1_000_000), 64, "f32", 8192, 0.1),
        # bags of about 20 lookups, bf16 rows
        _tables("tables-multihot", 8, (500_000, 500_000), 128, "bf16", 2048, 0.05, bag=20.0, alpha=1.2),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dispatch", "combine", "experts_bwd", "clip", "tables"])
    if op == "clip":
        c = _clip("", _logu(rng, 1, 1200), _logu(rng, 1000, 100_000_000),
                  rng.choice(["f32", "bf16", "f16", "bf16,f32", "f32,bf16,f16"]), rng.random() < 0.5,
                  rng.choice([0.1, 1.0, 1.0, 1e6]))
    elif op == "tables":
        multi = rng.random() < 0.4
        c = _tables("", rng.randint(1, 26), (_logu(rng, 10, 1000), _logu(rng, 2000, 1_000_000)),
                    rng.choice([8, 16, 20, 32, 64, 96, 128, rng.randint(1, 130)]), rng.choice(["f32", "f32", "bf16"]),
                    _logu(rng, 100, 8192 if not multi else 1024), round(rng.uniform(0.01, 0.5), 2),
                    bag=round(rng.uniform(1.5, 24.0), 2) if multi else 0.0, alpha=round(rng.uniform(1.05, 1.25), 3),
                    max_norm=rng.choice([0.1, 1.0, 10.0, 1e6]))
        while c["batch"] * c["tables"] * c["dim"] * max(1.0, c["bag"]) > 26 * 8192 * 64:
            c["batch"] = max(1, c["batch"] // 2)
    else:
        experts = _logu(rng, 2, 256)
        dim = rng.choice([64, 128, 256, 512, 1024, 2048, 4096, 5120, 8192]) if rng.random() < 0.7 else _logu(rng, 5, 6000)
        c = _route("", op, _logu(rng, 1, 16384), min(experts, rng.randint(1, 8)), experts, dim,
                   rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice([0.0, 0.0, 0.1, 0.5]),
                   rng.choice([0.0, 0.0, 1.0, 1.25]), rng.choice([1, 1, 16, 128]), rng.choice([0, 0, 8, 3]))
        while c["tokens"] * c["k"] * c["dim"] * (2 if op == "experts_bwd" else 1) > 4096 * 8 * 2048:
            c["tokens"] = max(1, c["tokens"] // 2)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
class State:
    """What a program keeps between calls: its buffers and, for the library, the handle."""

    def __init__(self, case):
        self.case, self.handle = case, None

    def __del__(self):
        if self.handle is not None and not sys.is_finalizing():
            torch.cuda.synchronize()
            self.handle.close()


def _gen(seed, word):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1_000_003 + word) & 0x7FFFFFFFFFFF)


def _capacity(c):
    return math.ceil(c["capacity"] * c["tokens"] * c["k"] / c["experts"]) if c["capacity"] else 0


def _n_rows(c):
    """Rows that hold any plan of the case: the experts' blocks, each rounded up to `align` rows."""
    n, e, cap, align = c["tokens"] * c["k"], c["experts"], _capacity(c), c["align"]
    most = -(-(min(cap, n) if cap else n) // align) * align
    return max(1, min(n + min(e, n) * (align - 1), e * most))


def _experts(c, seed):
    """int32 [tokens, k]: different experts in random order, -1 for padding tokens."""
    g, (t, e) = _gen(seed, 1), (c["tokens"], c["experts"])
    noise = -torch.log(-torch.log(torch.rand((t, e), generator=g, device="cuda").clamp(1e-7, 1 - 1e-6)))
    noise -= 0.5 * torch.log1p(torch.arange(e, device="cuda"))
    ids = torch.topk(noise, c["k"], dim=1).indices
    if c["drop"]:
        ids[torch.rand(t, generator=g, device="cuda") < c["drop"]] = -1
    return ids.to(torch.int32).contiguous()


def _rows(c, n, seed, word):
    """n rows of the case's type, `slack` elements further apart than they are long."""
    x = torch.randn((n, c["dim"] + c["slack"]), generator=_gen(seed, word), device="cuda").to(TYPES[c["dtype"]])
    return x[:, :c["dim"]]


def _empty(c, n):
    return torch.zeros((n, c["dim"] + c["slack"]), dtype=TYPES[c["dtype"]], device="cuda")[:, :c["dim"]]


def _weights(c, seed):
    w = torch.softmax(torch.randn((c["tokens"], c["k"]), generator=_gen(seed, 5), device="cuda"), 1)
    return w


def _sizes(c):
    """Elements of each tensor: spread over a factor of some thousand, a few tensors empty where there are many."""
    r = np.random.RandomState(c["tensors"])
    w = np.exp(r.uniform(0.0, 8.0, c["tensors"]))
    n = np.maximum(1, np.floor(w / w.sum() * c["total"])).astype(np.int64)
    if c["tensors"] > 100:
        n[r.randint(0, c["tensors"], 2)] = 0
    return n


def _places(c):
    """(type, offset, elements) of each tensor in the buffer of its type, and the buffers' lengths."""
    kinds, used, at = c["dtypes"].split(","), {}, []
    for i, n in enumerate(_sizes(c)):
        kind = kinds[i % len(kinds)]
        o = used.get(kind, 0)
        at.append((kind, o, int(n)))
        used[kind] = o + (int(n) if c["packed"] else -(-int(n) // 64) * 64)
    return at, used


def _gradients(c, seed):
    """The buffer of each type: gradients whose size differs by layer, zero between the tensors."""
    at, used = _places(c)
    bufs = {}
    for word, (kind, n) in enumerate(sorted(used.items())):
        g = _gen(seed, 20 + word)
        b = torch.randn(n, generator=g, device="cuda", dtype=TYPES[kind])
        parts = 64
        scale = torch.exp(torch.rand(parts, generator=g, device="cuda") * 4.0 - 7.0).to(TYPES[kind])
        b *= scale.repeat_interleave(-(-n // parts))[:n]
        bufs[kind] = b
    if not c["packed"]:
        for kind, o, n in at:
            bufs[kind][o + n:o + -(-n // 64) * 64] = 0
    return bufs


def _rows_per_table(c):
    t, lo, hi = c["tables"], c["rows_lo"], c["rows_hi"]
    return [max(1, round(lo * (hi / lo) ** (i / max(1, t - 1)))) for i in range(t)]


def _hot_per_table(c):
    return [max(1, math.ceil(n * c["hot"])) for n in _rows_per_table(c)]


def _lookups(c, seed):
    """bag_ptr [bags + 1], the bag of each lookup, its row among the hot rows and then the cold rows in use, and the
    number of the cold ones (int64)."""
    g, T, n_bags = _gen(seed, 7), c["tables"], c["batch"] * c["tables"]
    bags = torch.arange(n_bags, device="cuda")
    if c["bag"]:
        lens = torch.poisson(torch.full((n_bags,), c["bag"], device="cuda"), generator=_gen(0, 8)).long().clamp(max=64)
        ptr = torch.zeros(n_bags + 1, dtype=torch.int64, device="cuda")
        ptr[1:] = torch.cumsum(lens, 0)
        bag = torch.repeat_interleave(bags, lens)
    else:
        ptr, bag = torch.arange(n_bags + 1, device="cuda"), bags
    table = bag % T
    rows = torch.tensor(_rows_per_table(c), device="cuda")
    hot = torch.tensor(_hot_per_table(c), device="cuda")
    b = 1 - c["alpha"]
    h0, h1 = 0.5 ** b, (rows[table].double() + 0.5) ** b
    u = torch.rand(bag.numel(), generator=g, device="cuda", dtype=torch.float64)
    rank = torch.minimum(((h0 + u * (h1 - h0)) ** (1 / b) + 0.5).floor().long().clamp(min=1), rows[table]) - 1
    first, first_hot = torch.cumsum(rows, 0) - rows, torch.cumsum(hot, 0) - hot
    cold = rank >= hot[table]
    ids, at = torch.unique(torch.where(cold, first[table] + rank, -1), return_inverse=True)
    skip = int(ids.numel() and int(ids[0]) == -1)
    row = torch.where(cold, int(hot.sum()) + at - skip, first_hot[table] + rank)
    return ptr, bag, row, int(ids.numel()) - skip


def _table_values(c, n, seed):
    w = torch.rand((n, c["dim"]), generator=_gen(seed, 9), device="cuda") * 0.1 - 0.05
    return w.to(TYPES[c["dtype"]])


def _staging(c, cold, lookups):
    """The staging buffer: the cold rows in use, and room for as many as the lookups and the tables allow."""
    room = min(lookups, sum(_rows_per_table(c)) - sum(_hot_per_table(c)))
    return torch.cat([cold, cold.new_zeros((room - cold.shape[0], c["dim"]))])


def _dY(c, seed):
    return torch.randn((c["batch"] * c["tables"], c["dim"]), generator=_gen(seed, 10), device="cuda") * 0.01


def prepare(case, seed):
    c, s = case, State(case)
    i32 = dict(dtype=torch.int32, device="cuda")
    if own:
        from paper_2204_05436_amd import hotline as hl
        s.hl = hl
    if c["op"] == "clip":
        at, _ = _places(c)
        s.src = _gradients(c, seed)
        s.dst = {k: torch.zeros_like(v) for k, v in s.src.items()}
        s.norm = torch.zeros(1, device="cuda")
        if own:
            s.handle = hl.hl_create([1], 1, "f32", 1)
            s.list = hl.GradList([s.src[k][o:o + n] for k, o, n in at], [s.dst[k][o:o + n] for k, o, n in at])
            s.sq = torch.zeros(1, dtype=torch.float64, device="cuda")
            s.ws = torch.zeros(hl.hl_grad_workspace_bytes(), dtype=torch.uint8, device="cuda")
        return s
    if c["op"] == "tables":
        ptr, bag, row, n_cold = _lookups(c, seed)
        s.n_hot, s.L = sum(_hot_per_table(c)), int(row.numel())
        w = _table_values(c, s.n_hot + n_cold, seed)
        s.w_hot, s.staging = w[:s.n_hot].contiguous(), _staging(c, w[s.n_hot:], s.L)
        s.dY = _dY(c, seed)
        s.bag, s.row, s.norm = bag, row, torch.zeros(1, device="cuda")
        s.ptr, s.codes = ptr.to(torch.int32), row.to(torch.int32)
        if own:
            rows, hot = _rows_per_table(c), _hot_per_table(c)
            s.handle = hl.hl_create(rows, c["dim"], c["dtype"], s.n_hot)
            first = np.cumsum(rows) - rows
            ids = torch.cat([torch.arange(int(f), int(f) + n, **i32) for f, n in zip(first, hot)])
            hl.hl_set_hot(s.handle, ids, s.n_hot)
            s.sq = torch.zeros(1, dtype=torch.float64, device="cuda")
            s.ws = torch.zeros(hl.hl_workspace_bytes(s.handle, s.L, c["batch"] * c["tables"], c["batch"]),
                               dtype=torch.uint8, device="cuda")
        return s
    s.n_rows = _n_rows(c)
    s.experts = _experts(c, seed)
    n = c["tokens"] * c["k"]
    s.counts, s.offsets = torch.zeros(c["experts"], **i32), torch.zeros(c["experts"] + 1, **i32)
    s.pos, s.order = torch.zeros((c["tokens"], c["k"]), **i32), torch.full((s.n_rows,), -1, **i32)
    if c["op"] == "dispatch":
        s.x, s.rows = _rows(c, c["tokens"], seed, 2), _empty(c, s.n_rows)
    else:  # the plan that the forward left
        counts, offsets, pos, order = _plan(c, s.experts, s.n_rows)
        s.counts.copy_(counts), s.offsets.copy_(offsets), s.pos.copy_(pos.view_as(s.pos)), s.order.copy_(order)
        s.rows, s.w = _rows(c, s.n_rows, seed, 3), _weights(c, seed)
        s.out = _empty(c, c["tokens"])
        if c["op"] == "experts_bwd":
            s.dout, s.dgathered = _rows(c, c["tokens"], seed, 2), _rows(c, s.n_rows, seed, 4)
            s.drows, s.dw = _empty(c, s.n_rows), torch.zeros_like(s.w)
    if own:
        s.handle = hl.hl_create([1], 1, "f32", 1)
        s.route = hl.Route(c["tokens"], c["k"], c["experts"], s.counts, s.offsets, s.pos, s.order, capacity=_capacity(c),
                           align=c["align"])
        s.ws = torch.zeros(hl.hl_route_workspace_bytes(c["tokens"], c["k"], c["experts"]), dtype=torch.uint8,
                           device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms
def _plan(c, experts, n_rows):
    e = experts.view(-1).long()
    n, E, cap = e.numel(), c["experts"], _capacity(c)
    key = torch.where(e >= 0, e, E)
    at = torch.argsort(key, stable=True)
    found = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, key, torch.ones_like(key))
    i = torch.arange(n, device="cuda")
    rank = torch.empty_like(i)
    rank[at] = i - (torch.cumsum(found, 0) - found)[key[at]]
    counts = found[:E].clamp(max=cap) if cap else found[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum((counts + c["align"] - 1) // c["align"] * c["align"], 0)
    kept = (e >= 0) & (rank < cap) if cap else e >= 0
    pos = torch.where(kept, offsets[key] + rank, -1)
    order = torch.full((n_rows + 1,), -1, dtype=torch.int64, device="cuda")
    order[torch.where(kept, pos, n_rows)] = i
    i32 = torch.int32
    return counts.to(i32), offsets.to(i32), pos.to(i32), order[:n_rows].to(i32)


def _at_tokens(c, rows, pos):
    """[tokens, k, dim] in 32 bits: each assignment's row, zero where it has none."""
    p = pos.view(-1).long()
    v = rows[p.clamp(min=0)].float()
    return torch.where((p >= 0)[:, None], v, 0.0).view(c["tokens"], c["k"], c["dim"])


def _plain(s):
    c = s.case
    if c["op"] == "clip":
        norm = sum(v.float().square().sum(dtype=torch.float64) for v in s.src.values()).sqrt()
        scale = torch.where(norm > c["max_norm"], c["max_norm"] / norm, 1.0).float()
        return {k: (v.float() * scale).to(v.dtype) for k, v in s.src.items()}, norm.float().view(1)
    if c["op"] == "tables":
        rows, at = torch.unique(s.row, return_inverse=True)
        grad = torch.zeros((rows.numel(), c["dim"]), device="cuda").index_add_(0, at, s.dY[s.bag])
        norm = grad.square().sum(dtype=torch.float64).sqrt()
        step = LR * torch.where(norm > c["max_norm"], c["max_norm"] / norm, 1.0).float()
        hot = int((rows < s.n_hot).sum())
        for w, r, g in ((s.w_hot, rows[:hot], grad[:hot]), (s.staging, rows[hot:] - s.n_hot, grad[hot:])):
            w[r] = (w[r].float() - step * g).to(w.dtype)
        return s.w_hot, s.staging, norm.float().view(1)
    if c["op"] == "dispatch":
        counts, offsets, pos, order = _plan(c, s.experts, s.n_rows)
        token = order.clamp(min=0).long() // c["k"]
        s.rows.copy_(torch.where((order >= 0)[:, None], s.x[token], 0.0))
        return counts, offsets, pos.view_as(s.pos), order, s.rows
    if c["op"] == "combine":
        return ((_at_tokens(c, s.rows, s.pos) * s.w[:, :, None]).sum(1).to(s.rows.dtype),)
    dout = s.dout.float()
    dw = (_at_tokens(c, s.rows, s.pos) * dout[:, None, :]).sum(2)
    a = s.order.clamp(min=0).long()
    drows = torch.where((s.order >= 0)[:, None], dout[a // c["k"]] * s.w.view(-1)[a][:, None], 0.0).to(s.rows.dtype)
    return drows, dw, _at_tokens(c, s.dgathered, s.pos).sum(1).to(s.rows.dtype)


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state.case
    if not own:
        return _plain(s)
    hl, h = s.hl, s.handle
    if c["op"] == "clip":
        hl.hl_grad_sq(h, s.list, s.sq, s.ws)
        hl.hl_grad_clip(h, s.list, s.sq, c["max_norm"], s.norm)
        return s.dst, s.norm
    if c["op"] == "tables":
        B, T, cold = c["batch"], c["tables"], s.staging.shape[0]
        hl.hl_embbag_bwd_plan(h, cold, s.codes, s.ptr, B, T, s.L, None, None, B, s.ws)
        hl.hl_embbag_bwd_norm(h, cold, B, T, s.L, s.dY, s.sq, s.ws)
        hl.hl_embbag_bwd_clip(h, s.w_hot, s.staging, cold, B, T, s.L, s.sq, c["max_norm"], LR, s.ws, s.norm)
        return s.w_hot, s.staging, s.norm
    if c["op"] == "dispatch":
        hl.hl_route_plan(h, s.route, s.experts, s.ws)
        hl.hl_route_gather(h, s.route, s.x, s.rows)
        return s.counts, s.offsets, s.pos, s.order, s.rows
    if c["op"] == "combine":
        hl.hl_route_combine(h, s.route, s.rows, s.w, s.out)
        return (s.out,)
    hl.hl_route_combine_bwd(h, s.route, s.dout, s.rows, s.w, s.drows, s.dw)
    hl.hl_route_gather_bwd(h, s.route, s.dgathered, s.out)
    return s.drows, s.dw, s.out


# ------------------------------------------------------------------ what a pass cannot do without
def _kept(c):
    """Expected assignments that have a row (a capacity of c times the mean load drops some of the popular experts')."""
    n = c["tokens"] * c["k"] * (1 - c["drop"])
    if not c["capacity"]:
        return n
    p = 1.0 / np.sqrt(1.0 + np.arange(c["experts"]))
    return float(np.minimum(n * p / p.sum(), _capacity(c)).sum())


def work(case):
    c = case
    if c["op"] == "clip":
        size = {"f32": 4, "bf16": 2, "f16": 2}
        at, _ = _places(c)
        n = sum(x for _, _, x in at)
        return dict(bytes=2 * sum(size[k] * x for k, _, x in at) + 4, flops=3 * n)
    if c["op"] == "tables":
        n_bags = c["batch"] * c["tables"]
        L, used, b = n_bags * (c["bag"] or 1.0), 0.0, 1 - c["alpha"]
        for n in _rows_per_table(c):
            edge = (np.arange(n + 1) + 0.5) ** b
            p = (edge[:-1] - edge[1:]) / (edge[0] - edge[-1])
            used += float(-np.expm1(-(L / c["tables"]) * p).sum())
        row = c["dim"] * (4 if c["dtype"] == "f32" else 2)
        return dict(bytes=4 * L + 4 * (n_bags + 1) + 4 * n_bags * c["dim"] + 2 * used * row + 4,
                    flops=L * c["dim"] + 4 * used * c["dim"])
    n, kept = c["tokens"] * c["k"], _kept(c)
    row = c["dim"] * (4 if c["dtype"] == "f32" else 2)
    tokens, rows = c["tokens"] * row, kept * row
    if c["op"] == "dispatch":
        return dict(bytes=4 * n + 4 * n + 4 * kept + 8 * c["experts"] + tokens + rows, flops=0)
    if c["op"] == "combine":
        return dict(bytes=8 * n + rows + tokens, flops=2 * kept * c["dim"])
    return dict(bytes=12 * n + 2 * tokens + 3 * rows, flops=4 * kept * c["dim"])


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_plan(c, seed):
    e = _experts(c, seed).view(-1).cpu().numpy()
    cap, align, n_rows = _capacity(c), c["align"], _n_rows(c)
    counts, offsets = np.zeros(c["experts"], np.int32), np.zeros(c["experts"] + 1, np.int32)
    pos, order = np.full(e.size, -1, np.int32), np.full(n_rows, -1, np.int32)
    for x in range(c["experts"]):
        mine = np.flatnonzero(e == x)
        mine = mine[:cap] if cap else mine
        counts[x] = mine.size
        pos[mine] = offsets[x] + np.arange(mine.size)
        order[pos[mine]] = mine
        offsets[x + 1] = offsets[x] + (mine.size + align - 1) // align * align
    return counts, offsets, pos.reshape(c["tokens"], c["k"]), order


def _exact_sum(c, rows, pos, w=None):
    out = torch.zeros((c["tokens"], c["dim"]), dtype=torch.float64, device="cuda")
    for j in range(c["k"]):
        p = torch.from_numpy(pos[:, j]).cuda().long()
        t = (p >= 0).nonzero().view(-1)
        v = rows[p[t]].double()
        out.index_add_(0, t, v if w is None else v * w[t, j].double()[:, None])
    return out


def exact(case, seed):
    c = case
    if c["op"] == "clip":
        at, _ = _places(c)
        bufs = _gradients(c, seed)
        norm = math.sqrt(sum(float(bufs[k][o:o + n].double().pow(2).sum()) for k, o, n in at))
        scale = c["max_norm"] / norm if norm > c["max_norm"] else 1.0
        return {k: v.double() * scale for k, v in bufs.items()}, torch.tensor([norm], dtype=torch.float64)
    if c["op"] == "tables":
        _, bag, row, n_cold = _lookups(c, seed)
        n_hot = sum(_hot_per_table(c))
        w = _table_values(c, n_hot + n_cold, seed).double()
        grad = torch.zeros_like(w).index_add_(0, row, _dY(c, seed).double()[bag])
        norm = float(grad.pow(2).sum()) ** 0.5
        w -= LR * (c["max_norm"] / norm if norm > c["max_norm"] else 1.0) * grad
        return w[:n_hot], _staging(c, w[n_hot:], row.numel()), torch.tensor([norm], dtype=torch.float64)
    counts, offsets, pos, order = _exact_plan(c, seed)
    used = np.flatnonzero(order >= 0)
    a = torch.from_numpy(order[used]).cuda().long()
    at = torch.from_numpy(used).cuda()
    whole = torch.zeros((order.size, c["dim"]), dtype=torch.float64, device="cuda")
    if c["op"] == "dispatch":
        whole[at] = _rows(c, c["tokens"], seed, 2)[a // c["k"]].double()
        return counts, offsets, pos, order, whole
    rows, w = _rows(c, order.size, seed, 3), _weights(c, seed)
    if c["op"] == "combine":
        return (_exact_sum(c, rows, pos, w),)
    dout = _rows(c, c["tokens"], seed, 2)
    whole[at] = dout[a // c["k"]].double() * w.view(-1)[a].double()[:, None]
    dw = torch.zeros(w.numel(), dtype=torch.float64, device="cuda")
    for i in range(0, a.numel(), 16384):
        b = a[i:i + 16384]
        dw[b] = (dout[b // c["k"]].double() * rows[at[i:i + 16384]].double()).sum(1)
    return whole, dw.view(c["tokens"], c["k"]), _exact_sum(c, _rows(c, order.size, seed, 4), pos)
