"""HotPath.step with a bound on the norm refuses what it cannot clip before any part of the step runs: no gradient (the
norm would stay that of an earlier step), no bound, parts of the norm that the kernels could not read."""
import math
import types

import pytest
import torch

from paper_2204_05436_amd.runner import HotPath
from test_binding_devices import OnGpu


def step(**kw):
    """Whether the sequential step is reached."""
    ran = []
    dY = kw.pop("dY", OnGpu(torch.zeros(6, 4)))
    path = types.SimpleNamespace(w=types.SimpleNamespace(lr=0.1), h=types.SimpleNamespace(ptr=None, device=0, dim=4),
                                 _step_sequential=lambda *a: ran.append(a))
    batch = types.SimpleNamespace(n_samples=3, bps=2, n_lookups=9, n_bags=6, dY=dY)
    HotPath.step(path, batch, mode="sequential", **kw)
    return bool(ran)


def test_refused():
    parts = torch.zeros(3, dtype=torch.float64)
    for kw in [dict(max_norm=1.0, dY=None), dict(max_norm=-1.0), dict(max_norm=math.nan),
               dict(max_norm=1.0, norm_parts=parts), dict(max_norm=1.0, norm_parts=OnGpu(parts, 1)),
               dict(max_norm=1.0, norm_parts=OnGpu(parts.float())), dict(max_norm=1.0, norm_parts=OnGpu(parts[:0])),
               dict(max_norm=1.0, norm_parts=OnGpu(torch.zeros(6, dtype=torch.float64)[::2])),
               dict(norm_parts=OnGpu(parts))]:
        with pytest.raises(ValueError):
            step(**kw)


def test_taken():
    parts = OnGpu(torch.zeros(3, dtype=torch.float64))
    for kw in [dict(), dict(dY=None), dict(max_norm=0.0), dict(max_norm=math.inf), dict(max_norm=2, norm_parts=parts)]:
        assert step(**kw)
