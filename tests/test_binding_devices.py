"""The binding refuses tensors that a handle's kernels do not reach, before anything is launched: host memory (a GPU
fault otherwise), or another GPU's.  Without a GPU: the library is not called."""
import types

import pytest
import torch

from paper_2204_05436_amd import hotline as hl


class OnGpu:
    """A stand-in for a tensor of the same shape on a GPU."""

    def __init__(self, x, gpu=0):
        self.x, self.gpu, self.device = x, gpu, f"cuda:{gpu}"
        for a in ("dtype", "shape", "numel", "stride", "is_contiguous", "data_ptr", "element_size"):
            setattr(self, a, getattr(x, a))

    def get_device(self):
        return self.gpu

    def is_pinned(self):
        return False


class Pinned(OnGpu):
    def get_device(self):
        return -1

    def is_pinned(self):
        return True


class Reached(Exception):
    pass


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def lib():
        raise Reached  # (every check has passed)
    monkeypatch.setattr(hl, "lib", lib)


H = types.SimpleNamespace(ptr=None, device=0, dim=6)
I32, F32, F64, U8 = torch.int32, torch.float32, torch.float64, torch.uint8


def route(put, **kw):
    a = dict(counts=torch.zeros(3, dtype=I32), offsets=torch.zeros(4, dtype=I32), pos=torch.zeros(8, dtype=I32),
             order=torch.zeros(8, dtype=I32))
    a = {n: kw.get(n, put)(x) for n, x in a.items()}
    return hl.Route(4, 2, 3, n_rows=8, **a)


def calls():
    """Every call with its tensors: name -> (function of those tensors, the tensors)."""
    r = route(OnGpu)
    x, rows, w = torch.zeros(4, 6), torch.zeros(8, 6), torch.zeros(4, 2)
    sq, norm, ws = torch.zeros(1, dtype=F64), torch.zeros(1), torch.zeros(64, dtype=U8)
    grads = hl.GradList([OnGpu(torch.zeros(5))])
    return {
        "plan": (lambda e, ws: hl.hl_route_plan(H, r, e, ws, stream=0), [torch.zeros(8, dtype=I32), ws]),
        "gather": (lambda x, o: hl.hl_route_gather(H, r, x, o, stream=0), [x, rows]),
        "gather_bwd": (lambda d, x: hl.hl_route_gather_bwd(H, r, d, x, stream=0), [rows, x]),
        "combine": (lambda d, w, o: hl.hl_route_combine(H, r, d, w, o, stream=0), [rows, w, x]),
        "combine_bwd": (lambda d, o, w, dr, dw: hl.hl_route_combine_bwd(H, r, d, o, w, dr, dw, stream=0),
                        [x, rows, w, rows.clone(), w.clone()]),
        "grad_sq": (lambda s, ws: hl.hl_grad_sq(H, grads, s, ws, stream=0), [sq, ws]),
        "grad_clip": (lambda s, n: hl.hl_grad_clip(H, grads, s, 1.0, n, stream=0), [sq, norm]),
        "norm": (lambda d, s, ws: hl.hl_embbag_bwd_norm(H, 1, 2, 2, 9, d, s, ws, stream=0), [torch.zeros(4, 6), sq, ws]),
        "clip": (lambda w, st, s, ws, n: hl.hl_embbag_bwd_clip(H, w, st, 1, 2, 2, 9, s, 1.0, 0.1, ws, n, stream=0),
                 [rows, x, sq, ws, norm]),
    }


@pytest.mark.parametrize("name", calls())
def test_every_tensor_is_checked(name):
    f, ts = calls()[name]
    with pytest.raises(Reached):
        f(*map(OnGpu, ts))
    for i in range(len(ts)):
        put = lambda q: [(q if j == i else OnGpu)(t) for j, t in enumerate(ts)]
        with pytest.raises(ValueError):
            f(*put(lambda t: t))                # on the host
        with pytest.raises(ValueError):
            f(*put(lambda t: OnGpu(t, 1)))      # on another GPU
        with pytest.raises(Reached):
            f(*put(Pinned))                     # pinned host memory: every GPU reaches it
    with pytest.raises(ValueError):
        f(*(OnGpu(t, 1) for t in ts))


@pytest.mark.parametrize("which", ["counts", "offsets", "pos", "order"])
def test_plans_arrays(which):
    x, rows = OnGpu(torch.zeros(4, 6)), OnGpu(torch.zeros(8, 6))
    for put in (lambda t: t, lambda t: OnGpu(t, 1)):
        r = route(OnGpu, **{which: put})
        for f in (lambda: hl.hl_route_plan(H, r, OnGpu(torch.zeros(8, dtype=I32)), stream=0),
                  lambda: hl.hl_route_gather(H, r, x, rows, stream=0),
                  lambda: hl.hl_route_gather_bwd(H, r, rows, x, stream=0),
                  lambda: hl.hl_route_combine(H, r, rows, None, x, stream=0),
                  lambda: hl.hl_route_combine_bwd(H, r, x, None, None, rows, stream=0)):
            with pytest.raises(ValueError):
                f()


def test_gradients():
    on, sq, ws = OnGpu(torch.zeros(5)), OnGpu(torch.zeros(1, dtype=F64)), OnGpu(torch.zeros(64, dtype=U8))
    for bad in (hl.GradList([on, torch.zeros(3)]), hl.GradList([torch.zeros(3)]), hl.GradList([OnGpu(torch.zeros(3), 1)]),
                hl.GradList([on], [torch.zeros(5)]), hl.GradList([on, OnGpu(torch.zeros(3), 1)])):
        with pytest.raises(ValueError):
            hl.hl_grad_sq(H, bad, sq, ws, stream=0)
        with pytest.raises(ValueError):
            hl.hl_grad_clip(H, bad, sq, 1.0, stream=0)
    for good in (hl.GradList([]), hl.GradList([on]), hl.GradList([on, torch.zeros(0)]), hl.GradList([Pinned(torch.zeros(3)), on])):
        with pytest.raises(Reached):
            hl.hl_grad_sq(H, good, sq, ws, stream=0)


def test_norm_checks_the_gradient():
    """dY: n_samples * bags_per_sample rows of dim contiguous fp32 elements (the kernel reads it at every bag)."""
    sq, ws = OnGpu(torch.zeros(1, dtype=F64)), OnGpu(torch.zeros(64, dtype=U8))
    norm = lambda d: hl.hl_embbag_bwd_norm(H, 1, 2, 2, 9, d, sq, ws, stream=0)
    for bad in (torch.zeros(4, 5), torch.zeros(3, 6), torch.zeros(4, 6).double(), torch.zeros(4, 6).bfloat16(),
                torch.zeros(6, 4).t(), torch.zeros(4, 12)[:, :6]):
        with pytest.raises(ValueError):
            norm(OnGpu(bad))
    for good in (torch.zeros(4, 6), torch.zeros(24), torch.zeros(5, 6)):
        with pytest.raises(Reached):
            norm(OnGpu(good))
