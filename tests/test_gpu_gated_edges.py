"""Edges of the gated recurrent operators on the GPU: rates that no recurrence
has, infinite gates, rows behind the last sequence, very many sequences, and
weight gradients whose sums are exact."""
import math

import numpy as np
import pytest
import torch

from oracle import gated as G
from paper_2605_19150_amd import pdssm
from test_gpu_gated import DEV, Case, _all_ops, _check_bwd, _check_fwd, _near, _np

pytestmark = pytest.mark.gpu


def _dirty(*shapes):
    """Leaves memory of these sizes behind that holds NaN in every type."""
    keep = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for n in shapes for _ in range(4)]
    del keep


# ---- rates -----------------------------------------------------------------

BAD_RATES = [0.0, -0.0, -1.0, -1e-30, -3e38, math.inf, -math.inf, math.nan]


@pytest.mark.parametrize("dtype,C", [(torch.float32, 65), (torch.bfloat16, 65), (torch.bfloat16, 66)])
@pytest.mark.parametrize("bounds", [[0, 100], [0, 90, 400, 700]], ids=["one chunk", "chunks"])
def test_rates_that_are_not_positive_and_finite(bounds, dtype, C):
    """NaN in the rows of those channels, held ones among them, and in nothing else."""
    case = Case(bounds, C, dtype=dtype, wide=C % 2 == 1, seed=C)
    case.ga[5], case.ga[50] = -math.inf, -100.0
    good = case.rate
    y0, f0, s0, k0 = case.fwd(hold8=True)
    g0 = case.bwd(s0), case.bwd(s0, k0)
    case.rate = good.clone()
    bad = list(range(0, C, 8))
    for n, c in enumerate(bad):
        case.rate[c] = BAD_RATES[n % len(BAD_RATES)]
    rest = [c for c in range(C) if c not in bad]
    y, fin, saved, kept = case.fwd(hold8=True)
    for v, v0 in ((y, y0), (fin, f0)):
        assert torch.isnan(v[:, bad]).all() and torch.equal(v[:, rest], v0[:, rest])
    for a, b in zip(kept, k0):  # the form of the inputs knows no rate
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for got, want in zip((case.bwd(saved), case.bwd(saved, kept)), g0):
        for v, v0 in zip(got, want):
            assert torch.isnan(v[..., bad]).all() and torch.equal(v[..., rest], v0[..., rest])
    h = torch.randn(case.T, C, device=DEV)
    h0 = h.clone()
    _, ys = pdssm.gated_step(case.x, case.ga, case.gi, case.rate, h)
    _, y1 = pdssm.gated_step(case.x, case.ga, case.gi, good, h0)
    for v, v0 in ((h, h0), (ys, y1)):
        assert torch.isnan(v[:, bad]).all() and torch.equal(v[:, rest], v0[:, rest])
