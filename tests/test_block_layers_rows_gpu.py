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


def _centred_exact(x, gamma, beta, eps):
    """The forward pass where a row's mean may be far larger than its spread.

    Binary32: with m = D u max|x| the error of a first mean, s the mean and S the mean square of |x - mean|: the deviations from that first
    mean are rounded once, and their own mean, which takes the error out again, is off by e = (D + 3) u (s + m).  That is done where the
    mean is 64 times the spread or more (to be sure of that: 128 times as large as any deviation); elsewhere m stays as well.
    bfloat16, rows of one sign and of values within a factor of two of each other: a sum of up to 2^15 of them has at most 8 + 15 + 1
    bits and is exact, so that the first mean is off by its own two roundings, m = 2 u |mean|, and e = (D + 3) u s + m.
    x - mean is off by e and three roundings; the variance by (D + 4) u (S + m^2) from its sum, and by 2 m e + e^2 + 4 u m^2 from the
    square of what the mean is off."""
    bf16 = x.dtype == torch.bfloat16
    x, gm, bt = x.double(), gamma.double(), beta.double()
    mean = x.mean(1, keepdim=True)
    dev = x - mean
    var = (dev ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    xhat = dev * rstd
    y = xhat * gm + bt
    D = 80 if x.shape[1] <= 16384 else 4
    m = D * U * x.abs().amax(1, keepdim=True)
    far = mean ** 2 > 2.0 ** 14 * (dev.abs().amax(1, keepdim=True) ** 2 + eps)
    if bf16:
        m = torch.where(far, 2 * U * mean.abs(), m)
    e = (D + 3) * U * (dev.abs().mean(1, keepdim=True) + m)
    e = torch.where(far & (not bf16), e, e + m)
    spread = ((D + 4) * U * (var + m ** 2) + 2 * m * e + e ** 2 + 4 * U * m ** 2) / (var + eps)
    tol = gm.abs() * rstd * (e + 3 * U * (dev.abs() + m)) + (gm * xhat).abs() * (spread / 2 + spread ** 2 + 4 * U) \
        + U * ((gm * xhat).abs() + bt.abs() + y.abs())
    if bf16:    # of one value: beta, exactly
        tol = torch.where((dev == 0).all(1, keepdim=True), U * bt.abs(), tol)
    return y, mean, rstd, tol, e + 2 * U * mean.abs(), rstd * (spread / 2 + spread ** 2 + 4 * U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [24, 63, 100, 197, 255, 500, 768, 1000, 1025, 2560, 3001, 5000, 10000, 12281, 20000])
def test_norm_of_rows_far_from_zero(L, dtype):
    """Rows of one value give beta, whatever the value: the mean's rounding must not become a deviation.  A small spread on a large mean
    keeps the accuracy of the spread."""
    dt = base.DT[dtype]
    x = base._normal((10, L), torch.float32, "x", L)
    for r, v in enumerate((1e4, 12345.678, -1e6 / 3, 0.1, 0.0)):
        x[r] = v
    x[5] += 1e4
    x[6] = x[6] * 1e-2 + 1e4
    x[7] += 1e6
    x[8] = 3.0
    x[8, L // 2] = 4.0
    x = x.to(dt)
    gamma, beta = base._normal((L,), torch.float32, "gamma", L), base._normal((L,), torch.float32, "beta", L)
    y, stats = base._norm_fwd(x, gamma, beta, L)
    want, mean, rstd, tol, tm, tr = _centred_exact(x, gamma, beta, 1e-6)
    base._inside(y, want, tol + HALF[dt] * (want.abs() + tol), "y")
    base._inside(stats[:, :1], mean, tm, "mean")
    base._inside(stats[:, 1:], rstd, tr, "rstd")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lanes,L", [(lanes, L) for lanes, even, odd in TEAMS for L in (even, odd)] + [(512, 20000)])
def test_norm_rows_far_from_zero_among_others(lanes, L, dtype):
    """Every third row is far from zero.  The others must get the bits that they get without them, and the far rows theirs, in place too,
    over several rows of every team."""
    dt, rows = base.DT[dtype], _every_team_refills(lanes) if L < 16384 else 30
    plain = base._normal((rows, L), torch.float32, "x", rows, L)
    x = plain.clone()
    x[1::3] = x[1::3] * 1e-2 + 1e4
    x[4::9] = 12345.678
    x, plain = x.to(dt), plain.to(dt)
    gamma, beta = base._normal((L,), torch.float32, "gamma", L), base._normal((L,), torch.float32, "beta", L)
    y, stats = base._norm_fwd(x, gamma, beta, L)
    alone, alone_stats = base._norm_fwd(plain, gamma, beta, L)
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[1::3] = False
    assert torch.equal(y[other], alone[other]) and torch.equal(stats[other], alone_stats[other])
    far = x[~other]
    want, mean, rstd, tol, tm, tr = _centred_exact(far, gamma, beta, 1e-6)
    base._inside(y[~other], want, tol + HALF[dt] * (want.abs() + tol), "y")
    base._inside(stats[~other][:, :1], mean, tm, "mean")
    base._inside(stats[~other][:, 1:], rstd, tr, "rstd")
    again = torch.empty_like(stats)
    s2a.s2a_layernorm_fwd(x, gamma, beta, x, again, L, 1e-6)
    base._done()
    assert torch.equal(x, y) and torch.equal(again, stats)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [5, 24, 63, 197, 768, 1000, 1025, 3001, 10000, 20000])
def test_norm_statistics_of_infinite_rows(L, dtype):
    """The mean of a row with an infinity is that infinity, of both it is NaN; the rows around it keep their bits."""
    dt = base.DT[dtype]
    plain = base._normal((6, L), dt, "x", L)
    x = plain.clone()
    x[1, L // 2] = float("inf")
    x[2, L - 1] = float("-inf")
    x[3, 0], x[3, L - 1] = float("inf"), float("-inf")
    x[4, L // 3] = float("nan")
    y, stats = base._norm_fwd(x, None, None, L)
    alone, alone_stats = base._norm_fwd(plain, None, None, L)
    assert float(stats[1, 0]) == float("inf") and float(stats[2, 0]) == float("-inf")
    assert bool(torch.isnan(stats[3:5, 0]).all()) and bool(torch.isnan(stats[1:5, 1]).all()) and bool(torch.isnan(y[1:5]).all())
    for r in (0, 5):
        assert torch.equal(y[r], alone[r]) and torch.equal(stats[r], alone_stats[r])
