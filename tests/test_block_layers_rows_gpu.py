"""Layer norm over many rows of every team width, and over rows of tens of millions of elements.

Tolerances are those of test_block_layers_gpu.py, with the additions that a term passes through counted for the rows at hand:
a column's sum over n rows by T teams of one CTA each at least has ceil(n / T) in a thread, T per CTA <= 32, at most 444 / 32 + 1
partials and 5 shuffle steps; a long row's sums are held in 64 bits, and rounded to binary32 once."""
import math

import pytest
import torch

import test_block_layers_gpu as base
from paper_2503_08154_b200 import binding as s2a

pytestmark = pytest.mark.gpu

U, HALF = base.U, base.HALF

# lanes of a team and the row lengths it takes: one on the 16-byte grid, one odd
TEAMS = [(8, 40, 63), (16, 72, 121), (32, 200, 255), (32, 400, 511), (32, 600, 761), (64, 1000, 1017), (64, 1200, 1025), (128, 1600, 2039),
         (128, 2560, 3001), (256, 3200, 4089), (256, 5000, 6137), (512, 6400, 8185), (512, 10000, 12281), (512, 12296, 16377)]


def _every_team_refills(lanes):
    """Rows enough for each team to take more than its ring holds: at most 148 SMs x 4 CTAs, at most 4 rows in flight."""
    teams = 148 * (4 * 256 // lanes if lanes <= 256 else 1)
    return 5 * teams + 3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lanes,L", [(lanes, L) for lanes, even, odd in TEAMS for L in (even, odd)])
def test_norm_rings_are_refilled(lanes, L, dtype):
    dt, rows = base.DT[dtype], _every_team_refills(lanes)
    x = base._normal((rows, L), dt, "x", rows, L) + base._normal((rows, 1), dt, "off", rows, L)
    gamma, beta = base._normal((L,), torch.float32, "gamma", L) * 0.3 + 1, base._normal((L,), torch.float32, "beta", L)
    y, stats = base._norm_fwd(x, gamma, beta, L)
    want, mean, rstd, tol, tm, tr = base._norm_exact(x, gamma, beta, 1e-6)
    base._inside(stats[:, :1], mean, tm + U * mean.abs(), "mean")
    base._inside(stats[:, 1:], rstd, tr, "rstd")
    base._inside(y, want, tol + HALF[dt] * (want.abs() + tol), "y")
    del want, tol
    # gradients of whole numbers: the columns' sums of them are exact in any order, so that no row may be lost or counted twice
    g = torch.randint(-8, 9, (rows, L), generator=base._gen("g", rows, L), device="cuda").to(dt)
    assert 8 * rows < 2 ** 24
    gin, dgamma, dbeta = torch.empty_like(x), torch.empty(L, device="cuda"), torch.empty(L, device="cuda")
    scratch = torch.empty(s2a.layernorm_scratch_bytes(rows, L), dtype=torch.uint8, device="cuda").fill_(0xFF)
    s2a.s2a_layernorm_bwd(g, x, gamma, stats, gin, dgamma, dbeta, scratch, L)
    base._done()
    dx, dg, db, tol, _, _ = base._norm_bwd_tolerance(g, x, gamma, stats)
    base._inside(gin, dx, tol + HALF[dt] * (dx.abs() + tol), "grad_in")
    del dx, tol
    assert torch.equal(dbeta.double(), db)
    teams = 144 * (256 // lanes if lanes <= 256 else 1)      # odd rows: whole periods of eight shifts
    Dc = math.ceil(rows / teams) + 32 + 15 + 5
    mass = (g.double() * (x.double() - stats[:, :1].double()) * stats[:, 1:].double()).abs().sum(0)
    base._inside(dgamma, dg, (Dc + 4) * U * mass + U * dg.abs(), "grad_gamma")
    # in place, every one of the rows: the same bits
    for target in (0, 1):
        pair = [g.clone(), x.clone()]
        s2a.s2a_layernorm_bwd(pair[0], pair[1], gamma, stats, pair[target], None, None, None, L)
        base._done()
        assert torch.equal(pair[target], gin)
    again = torch.empty_like(stats)
    s2a.s2a_layernorm_fwd(x, gamma, beta, x, again, L, 1e-6)
    base._done()
    assert torch.equal(x, y) and torch.equal(again, stats)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_rows_of_tens_of_millions(dtype, monkeypatch):
    """A thread has some sixty thousand terms of a row.  Of one sign and nearly alike, as here, they would all be rounded the same way
    in a binary32 sum."""
    rows, L, dt = 3, 30_000_001, base.DT[dtype]
    x = (1.1 + base._normal((rows, L), torch.float32, "x", L) * 2.0 ** -6).to(dt)
    x[2] = 1.1
    g = (1.7 + base._normal((rows, L), torch.float32, "g", L) * 2.0 ** -6).to(dt)
    monkeypatch.setattr(base, "_depth", lambda row_len: 4)   # a sum's rounding and those of its terms
    _, stats = base._check_norm_fwd(x, None, None, L)
    base._check_norm_bwd(g, x, None, stats, L)
