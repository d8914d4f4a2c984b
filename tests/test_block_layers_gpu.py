"""GPU parity of layer norm, dropout and the relative position bias against plain 64-bit forms.

Tolerances, with u = 2^-24 (half a step of binary32) and h the half step of the output type (2^-8 for bfloat16, u
for binary32).  A sum of binary32 terms in which no term passes through more than D additions is off by at most
D u sum|terms|; a row's sums have D <= 80 in registers (32 terms a lane, 5 shuffle steps, 16 warps, and the merge), and
D <= row_len / 512 + 40 for rows of more than 16384 elements.  A column's sum over n rows has D <= ceil(n / 296) + 64: at
least 296 teams share the rows (or each has one), 8 teams and 296 / 8 + 8 partials are added after that; for the long
rows a thread takes at most 64 rows before that, or n / 296.

* layer norm forward: the mean is off by at most m = D u mean|x|; x - mean is rounded once; the variance has the relative
  error (D + 4) u + (m rstd)^2, its root half of that, the reciprocal root two roundings more; then two products and
  one sum: |dy| <= |gamma| rstd (m + u |x - mean|) + |gamma xhat| ((D + 4) u / 2 + (m rstd)^2 / 2 + 4 u) + u (|gamma xhat| +
  |beta| + |y|) + h |y|.
* layer norm backward (mean and rstd are inputs): see `_norm_bwd_tolerance`.
* dropout: the scale is rounded once and the product once, with the residual one more: 2 u |x scale| + u |y| + h |y|.
* bias forward: u |y| + h |y|.  The table's gradient: with whole-number gradients every sum is exact, and the result is
  the rounding of the true sum; with others D <= batch + 2048 at the sizes tested.
Results below the normal range may be flushed: + 2^-126.
"""
import math

import numpy as np
import pytest
import torch

import parity_util as pu
from paper_2503_08154_b200 import binding as s2a

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -126
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def _gen(*key):
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * ord(c) for i, c in enumerate(repr(key))))


def _normal(shape, dtype, *key, scale=1.0):
    return (torch.randn(shape, generator=_gen(*key), device="cuda") * scale).to(dtype)


def _inside(got, want, tol, what):
    got, want, tol = got.double(), want.double(), tol.double() + TINY
    bad = ~((got - want).abs() <= tol)
    if bool(bad.any()):
        at = torch.nonzero(bad)[0].tolist()
        i = tuple(at)
        raise AssertionError("%s: %d of %d outside tolerance, first at %s: got %r want %r tol %r"
                             % (what, int(bad.sum()), bad.numel(), at, float(got[i]), float(want[i]), float(tol.expand_as(got)[i])))


def _guarded(shape, dtype):
    n = int(np.prod(shape))
    g = pu.Guarded(n * dtype.itemsize)
    return g, g.view(dtype).view(shape)


def _done():
    torch.cuda.synchronize()
    assert s2a.s2a_device_error() == 0


# ------------------------------------------------------------------------------------------ layer norm
def _depth(L):
    return 80 if L <= 16384 else L / 512 + 40


def _norm_exact(x, gamma, beta, eps):
    x = x.double()
    L = x.shape[1]
    mean = x.mean(1, keepdim=True)
    rstd = (((x - mean) ** 2).mean(1, keepdim=True) + eps) ** -0.5
    xhat = (x - mean) * rstd
    gm = torch.ones(L, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    bt = torch.zeros(L, dtype=torch.float64, device="cuda") if beta is None else beta.double()
    y = xhat * gm + bt
    D = _depth(L)
    m = D * U * x.abs().mean(1, keepdim=True)
    spread = (D + 4) * U + (m * rstd) ** 2
    tol = gm.abs() * rstd * (m + U * (x - mean).abs()) + (gm * xhat).abs() * (spread / 2 + 4 * U) \
        + U * ((gm * xhat).abs() + bt.abs() + y.abs())
    return y, mean, rstd, tol, m, rstd * (spread / 2 + 3 * U)


def _norm_fwd(x, gamma, beta, L, eps=1e-6):
    n = x.numel() // L
    gy, y = _guarded((n, L), x.dtype)
    gs, stats = _guarded((n, 2), torch.float32)
    s2a.s2a_layernorm_fwd(x, gamma, beta, y, stats, L, eps)
    _done()
    gy.check("y"), gs.check("stats")
    return y, stats


def _check_norm_fwd(x, gamma, beta, L, eps=1e-6):
    y, stats = _norm_fwd(x, gamma, beta, L, eps)
    want, mean, rstd, tol, tm, tr = _norm_exact(x.reshape(-1, L), gamma, beta, eps)
    _inside(stats[:, :1], mean, tm + U * mean.abs(), "mean")
    _inside(stats[:, 1:], rstd, tr, "rstd")
    _inside(y, want, tol + HALF[x.dtype] * (want.abs() + tol), "y")
    return y, stats


def _norm_bwd_exact(g, x, gamma, stats):
    g, x, st = g.double(), x.double(), stats.double()
    L = x.shape[1]
    gm = torch.ones(L, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    mean, rstd = st[:, :1], st[:, 1:]
    xhat = (x - mean) * rstd
    a = g * gm
    m1, m2 = a.mean(1, keepdim=True), (a * xhat).mean(1, keepdim=True)
    dx = rstd * (a - m1 - xhat * m2)
    return dx, (g * xhat).sum(0), g.sum(0), a, xhat, m1, m2


def _norm_bwd_tolerance(g, x, gamma, stats):
    """xhat has two roundings, a one; the sums D additions over that; then, for each term of a - m1 - xhat m2, at most six
    more (1 / row_len rounded, the products, the two sums, rstd)."""
    dx, dg, db, a, xhat, m1, m2 = _norm_bwd_exact(g, x, gamma, stats)
    L, n = x.shape[1], x.shape[0]
    D = _depth(L)
    rstd = stats.double()[:, 1:]
    e1 = (D + 3) * U * a.abs().mean(1, keepdim=True)
    e2 = (D + 5) * U * (a * xhat).abs().mean(1, keepdim=True)
    tol = rstd.abs() * (e1 + xhat.abs() * e2 + 6 * U * (a.abs() + m1.abs() + (xhat * m2).abs()))
    Dc = math.ceil(n / 296) + 64 + (64 if L > 16384 else 0)
    tg = (Dc + 4) * U * (g.double() * xhat).abs().sum(0)
    tb = (Dc + 1) * U * g.double().abs().sum(0)
    return dx, dg, db, tol, tg, tb


def _check_norm_bwd(g, x, gamma, stats, L, weights=torch.float32):
    n = x.numel() // L
    gi, gin = _guarded((n, L), x.dtype)
    gg, dgamma = _guarded((L,), weights)
    gb, dbeta = _guarded((L,), weights)
    gs, scratch = _guarded((s2a.layernorm_scratch_bytes(n, L),), torch.uint8)
    s2a.s2a_layernorm_bwd(g, x, gamma, stats, gin, dgamma, dbeta, scratch, L)
    _done()
    for guard, what in ((gi, "grad_in"), (gg, "grad_gamma"), (gb, "grad_beta"), (gs, "scratch")):
        guard.check(what)
    dx, dg, db, tol, tg, tb = _norm_bwd_tolerance(g.reshape(-1, L), x.reshape(-1, L), gamma, stats)
    _inside(gin, dx, tol + HALF[x.dtype] * (dx.abs() + tol), "grad_in")
    _inside(dgamma, dg, tg + HALF[weights] * (dg.abs() + tg), "grad_gamma")
    _inside(dbeta, db, tb + HALF[weights] * (db.abs() + tb), "grad_beta")
    frozen = torch.empty_like(gin)
    s2a.s2a_layernorm_bwd(g, x, gamma, stats, frozen, None, None, None, L)
    _done()
    assert torch.equal(frozen, gin) or torch.allclose(frozen.double(), gin.double(), rtol=0, atol=0, equal_nan=True)
    return gin, dgamma, dbeta


# one piece and many, every team width's first and last row length, odd lengths, a long row
NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (4, 8), (9, 31), (7, 33), (8, 64), (300, 96), (2, 255), (17, 256), (5, 257), (13, 512),
               (11, 513), (197, 768), (64, 776), (6, 1000), (5, 1024), (9, 1025), (4, 1032), (33, 1280), (3, 1537), (3, 2048),
               (2, 2049), (7, 3333), (5, 4096), (3, 4097), (2, 6144), (3, 8192), (2, 8193), (2, 12289), (3, 16384), (2, 16385),
               (3, 20000), (1, 65537)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,L", NORM_SHAPES)
def test_norm_forward_and_backward(rows, L, dtype):
    dt, wt = (DT[dtype], DT["f32"] if (rows + L) % 2 else DT["bf16"])
    x = _normal((rows, L), dt, "x", rows, L) * 1.5 + _normal((rows, 1), dt, "off", rows, L)
    gamma, beta = _normal((L,), wt, "gamma", L) * 0.3 + 1, _normal((L,), wt, "beta", L)
    _, stats = _check_norm_fwd(x, gamma, beta, L)
    _check_norm_bwd(_normal((rows, L), dt, "g", rows, L), x, gamma, stats, L, wt)


@pytest.mark.parametrize("rows,L", [(5000, 768), (2500, 1025), (1300, 4096), (3001, 40), (700, 577), (400, 17000)])
def test_norm_backward_over_many_rows(rows, L):
    for dt in (torch.bfloat16, torch.float32):
        x = _normal((rows, L), dt, "x", rows, L)
        _, stats = _norm_fwd(x, None, None, L)
        _check_norm_bwd(_normal((rows, L), dt, "g", rows, L), x, None, stats, L)


def test_norm_beta_gradient_of_whole_numbers_is_exact_and_repeats():
    rows, L = 4001, 1000
    g = torch.randint(-8, 9, (rows, L), generator=_gen("int"), device="cuda").float()
    x = _normal((rows, L), torch.float32, "x")
    _, stats = _norm_fwd(x, None, None, L)
    first = _check_norm_bwd(g, x, None, stats, L)
    assert torch.equal(first[2], g.sum(0))
    for _ in range(3):
        again = _check_norm_bwd(g, x, None, stats, L)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("missing", ["gamma", "beta", "both", "stats"])
def test_norm_optional_arguments(missing):
    rows, L = 37, 200
    x = _normal((rows, L), torch.bfloat16, "x")
    gamma = None if missing in ("gamma", "both") else _normal((L,), torch.float32, "gamma")
    beta = None if missing in ("beta", "both") else _normal((L,), torch.float32, "beta")
    if missing == "stats":
        y = torch.empty_like(x)
        s2a.s2a_layernorm_fwd(x, gamma, beta, y, None, L, 1e-6)
        _done()
        assert torch.equal(y, _norm_fwd(x, gamma, beta, L)[0])
        return
    _, stats = _check_norm_fwd(x, gamma, beta, L)
    g = _normal((rows, L), torch.bfloat16, "g")
    full = _check_norm_bwd(g, x, gamma, stats, L)
    scratch = torch.empty(s2a.layernorm_scratch_bytes(rows, L), dtype=torch.uint8, device="cuda")
    for which in (1, 2):    # one of the two weights frozen
        out = [torch.empty_like(x), torch.full((L,), 7.0, device="cuda"), torch.full((L,), 7.0, device="cuda")]
        grads = [out[i] if i != which else None for i in (1, 2)]
        s2a.s2a_layernorm_bwd(g, x, gamma, stats, out[0], grads[0], grads[1], scratch, L)
        _done()
        assert torch.equal(out[0], full[0]) and torch.equal(out[3 - which], full[3 - which])
        assert bool((out[which] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,stride,offset", [(64, 64 * 5, 0), (768, 768 * 197, 768), (40, 48, 3), (100, 104, 1), (33, 35, 0),
                                             (1024, 1032, 8), (2000, 2001, 0), (17000, 17003, 2)])
def test_norm_rows_of_a_larger_tensor(L, stride, offset, dtype):
    rows, dt = 6, DT[dtype]
    buf = _normal((rows * stride + offset,), dt, "buf", L, stride)
    x = buf[offset:].view(rows, stride)[:, :L]
    gamma, beta = _normal((L,), torch.float32, "gamma"), _normal((L,), torch.float32, "beta")
    plain_y, plain_stats = _check_norm_fwd(x.contiguous(), gamma, beta, L)
    out = torch.full((rows * stride + offset,), 3.0, dtype=dt, device="cuda")
    y = out[offset:].view(rows, stride)[:, :L]
    stats = torch.empty((rows, 2), device="cuda")
    s2a.s2a_layernorm_fwd(x, gamma, beta, y, stats, L, 1e-6)
    _done()
    # a row's sums may run in another order when the rows are not aligned: the same tolerance, not the same bits
    want, _, _, tol, tm, tr = _norm_exact(x, gamma, beta, 1e-6)
    _inside(y, want, tol + HALF[dt] * (want.abs() + tol), "strided y")
    untouched = torch.ones(rows * stride + offset, dtype=torch.bool, device="cuda")
    untouched[offset:].view(rows, stride)[:, :L] = False
    assert bool((out[untouched] == 3.0).all()), "elements between the rows were written"
    # backward with three different strides, into a slice
    g = _normal((rows, L + 5), dt, "g", L)[:, 2:2 + L]
    out.fill_(3.0)
    dgamma, dbeta = torch.empty(L, device="cuda"), torch.empty(L, device="cuda")
    scratch = torch.empty(s2a.layernorm_scratch_bytes(rows, L), dtype=torch.uint8, device="cuda")
    s2a.s2a_layernorm_bwd(g, x, gamma, plain_stats, y, dgamma, dbeta, scratch, L)
    _done()
    dx, dg, db, tol, tg, tb = _norm_bwd_tolerance(g, x, gamma, plain_stats)
    _inside(y, dx, tol + HALF[dt] * (dx.abs() + tol), "strided grad_in")
    _inside(dgamma, dg, tg + U * dg.abs(), "grad_gamma")
    _inside(dbeta, db, tb + U * db.abs(), "grad_beta")
    assert bool((out[untouched] == 3.0).all())


@pytest.mark.parametrize("rows,L", [(50, 768), (50, 777), (20, 5000), (3, 17000)])
def test_norm_in_place(rows, L):
    for dt in (torch.float32, torch.bfloat16):
        x, g = _normal((rows, L), dt, "x"), _normal((rows, L), dt, "g")
        gamma = _normal((L,), dt, "gamma")
        y, stats = _norm_fwd(x, gamma, gamma, L)
        here = x.clone()
        s2a.s2a_layernorm_fwd(here, gamma, gamma, here, stats, L, 1e-6)
        assert torch.equal(here, y)
        gin, dgamma, dbeta = _check_norm_bwd(g, x, gamma, stats, L, dt)
        scratch = torch.empty(s2a.layernorm_scratch_bytes(rows, L), dtype=torch.uint8, device="cuda")
        for target in (0, 1):
            pair = [g.clone(), x.clone()]
            dg, db = torch.empty_like(gamma), torch.empty_like(gamma)
            s2a.s2a_layernorm_bwd(pair[0], pair[1], gamma, stats, pair[target], dg, db, scratch, L)
            _done()
            assert torch.equal(pair[target], gin) and torch.equal(dg, dgamma) and torch.equal(db, dbeta)
            assert torch.equal(pair[1 - target], (g, x)[1 - target])


def test_norm_constant_large_and_non_finite_rows():
    L = 768
    x = _normal((6, L), torch.float32, "x")
    x[0] = 3.0                       # no variance: y = beta, whatever the rounding of the mean leaves over
    x[1] = x[1] * 1e-3 + 1e4         # a small spread on a large mean: a difference of squares would lose it all
    x[2] *= 1e15
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    gamma, beta = _normal((L,), torch.float32, "gamma"), _normal((L,), torch.float32, "beta")
    y, stats = _norm_fwd(x, gamma, beta, L)
    want, mean, rstd, tol, tm, tr = _norm_exact(x, gamma, beta, 1e-6)
    fine = [0, 1, 2, 5]
    _inside(y[fine], want[fine], (tol + U * want.abs())[fine], "y")
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[4]).all())     # as the formula has it
    assert bool(torch.isfinite(y[fine]).all()), "a row's NaN must stay in its row"


def test_norm_without_rows():
    x = torch.empty((0, 48), dtype=torch.bfloat16, device="cuda")
    st = torch.empty((0, 2), device="cuda")
    gamma = torch.ones(48, device="cuda")
    s2a.s2a_layernorm_fwd(x, gamma, gamma, x.clone(), st, 48, 1e-6)
    dg, db = torch.full((48,), 7.0, device="cuda"), torch.full((48,), 7.0, device="cuda")
    scratch = torch.empty(s2a.layernorm_scratch_bytes(0, 48), dtype=torch.uint8, device="cuda")
    s2a.s2a_layernorm_bwd(x, x.clone(), gamma, st, x.clone(), dg, db, scratch, 48)
    _done()
    assert bool((dg == 0).all()) and bool((db == 0).all())


def test_norm_rows_beyond_32_bit_offsets():
    L, stride = 1000, (1 << 31) + 16
    buf = torch.empty(2 * stride + L, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, L), (stride, 1))
    x.copy_(_normal((3, L), torch.bfloat16, "far"))
    _check_norm_fwd(x, None, None, L)
    near = x.contiguous()
    _, stats = _norm_fwd(near, None, None, L)
    g = _normal((3, L), torch.bfloat16, "g")
    want = _check_norm_bwd(g, near, None, stats, L)
    got = [torch.empty_like(t) for t in want]
    scratch = torch.empty(s2a.layernorm_scratch_bytes(3, L), dtype=torch.uint8, device="cuda")
    s2a.s2a_layernorm_bwd(g, x, None, stats, got[0], got[1], got[2], scratch, L)
    _done()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_norm_gradient_is_the_forward_pass_differences():
    """<grad, v> against the difference quotient of the kernels' own forward pass, in binary32.  What the quotient may be
    off by: its truncation (computed in 64 bits) and the forward pass's tolerance at the two points over 2 h; and the
    gradient by its own tolerance."""
    rows, L, h = 12, 301, 2.0 ** -6
    x, w = _normal((rows, L), torch.float32, "x"), _normal((rows, L), torch.float32, "w")
    gamma, beta = _normal((L,), torch.float32, "gamma") * 0.3 + 1, _normal((L,), torch.float32, "beta")
    y, stats = _norm_fwd(x, gamma, beta, L)
    gin, dgamma, dbeta = _check_norm_bwd(w, x, gamma, stats, L)
    for k, grad in enumerate((gin, dgamma, dbeta)):
        args = [x, gamma, beta]
        v = torch.sign(_normal(args[k].shape, torch.float32, "v", k))
        points, quotient, allowed, exact = [], 0.0, 0.0, 0.0
        for s in (1, -1):
            moved = list(args)
            moved[k] = args[k] + s * h * v
            out, _ = _norm_fwd(moved[0], moved[1], moved[2], L)
            want, _, _, tol, _, _ = _norm_exact(moved[0], moved[1], moved[2], 1e-6)
            quotient += s * float((out.double() * w.double()).sum()) / (2 * h)
            exact += s * float((want * w.double()).sum()) / (2 * h)
            allowed += float(((tol + U * want.abs() + TINY) * w.double().abs()).sum()) / (2 * h)
        dx, dg, db, tol, tg, tb = _norm_bwd_tolerance(w, x, gamma, stats)
        truth, own = ((dx, tol + U * dx.abs()), (dg, tg + U * dg.abs()), (db, tb + U * db.abs()))[k]
        # the kept (mean, rstd) are rounded: that moves the 64-bit gradient by at most their relative error
        slope = float((truth * v.double()).sum())
        allowed += abs(slope - exact) + float(own.sum())
        assert abs(float((grad.double() * v.double()).sum()) - quotient) <= allowed


# ------------------------------------------------------------------------------------------ dropout
def _philox(counter, key):
    """Philox4x32-10 in Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def _bits(n, seed, offset, site, first=0):
    """The 16 bits of elements first .. first + n - 1 (first a multiple of 8)."""
    count = (offset + site) % (1 << 64)
    out = []
    for b in range(first // 8, (first + n + 7) // 8):
        words = _philox([b & 0xFFFFFFFF, b >> 32, count & 0xFFFFFFFF, count >> 32], [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF])
        for w in words:
            out += [w & 0xFFFF, w >> 16]
    return np.array(out[:n])


def _rng(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def test_philox_known_answers():
    # the generator's published vectors: all zeros, all ones, and the digits of pi
    assert _philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert _philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert _philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def _check_dropout(n, p, dtype, residual, seed=0x123456789ABCDEF, offset=77, site=5):
    dt = DT[dtype]
    x = _normal((n,), dt, "x", n)
    r = _normal((n,), dt, "r", n) if residual else None
    guard, y = _guarded((n,), dt)
    s2a.s2a_dropout_fwd(x, r, y, _rng(seed, offset), site, p)
    _done()
    guard.check("y")
    T = s2a.dropout_threshold(p)
    keep = torch.from_numpy(_bits(n, seed, offset, site) >= T).cuda()
    part = torch.where(keep, x.double(), 0.0) * (65536 / (65536 - T) if T < 65536 else 0.0)
    want = part if r is None else part + r.double()
    _inside(y, want, 2 * U * part.abs() + (U + HALF[dt]) * want.abs() * (1 + 2 * U), "dropout")
    if r is None:
        if n:
            assert bool(((y == 0) == ~(keep & (x != 0))).all())
        gin = torch.empty_like(x)
        s2a.s2a_dropout_bwd(x, gin, _rng(seed, offset), site, p)
        _done()
        assert torch.equal(gin, y), "the backward pass must draw the forward pass's mask"
    return keep


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [0, 1, 2, 7, 8, 9, 15, 16, 63, 255, 1000, 2047, 2048, 2049, 20011, 77 * 1024 + 5])
def test_dropout_mask_and_values(n, dtype):
    for residual in (False, True):
        for p in (0.1, 0.5):
            _check_dropout(n, p, dtype, residual)


@pytest.mark.parametrize("p", [0.0, 1e-9, 2.0 ** -16, 0.25, 0.9, 1 - 2.0 ** -16, 1 - 1e-9, 1.0])
def test_dropout_probabilities(p):
    for dtype in ("f32", "bf16"):
        for residual in (False, True):
            _check_dropout(4103, p, dtype, residual)


@pytest.mark.parametrize("seed,offset,site", [(0, 0, 0), (-1, -1, 0), (1 << 62, (1 << 32) - 1, 1), (5, -1, 1), (7, 1 << 40, (1 << 64) - 3),
                                              (-(1 << 63), 3, -4)])
def test_dropout_keys_and_counters(seed, offset, site):
    # 64-bit words as a user stores them, signed; the offset and the site add modulo 2^64
    n = 500
    x = torch.ones(n, device="cuda")
    y = torch.empty_like(x)
    s2a.s2a_dropout_fwd(x, None, y, _rng(seed, offset), site, 0.5)
    _done()
    want = _bits(n, seed % (1 << 64), offset % (1 << 64), site % (1 << 64)) >= 32768
    assert np.array_equal(y.cpu().numpy() != 0, want)


def test_dropout_leaves_nothing_of_dropped_infinities():
    n = 8192
    for dt in (torch.float32, torch.bfloat16):
        keep = torch.from_numpy(_bits(n, 9, 8, 7) >= s2a.dropout_threshold(0.5)).cuda()
        for bad in (float("inf"), float("-inf"), float("nan")):
            x = torch.ones(n, dtype=dt, device="cuda")
            x[~keep] = bad
            y = torch.empty_like(x)
            s2a.s2a_dropout_fwd(x, None, y, _rng(9, 8), 7, 0.5)
            s2a.s2a_dropout_fwd(x, x.new_ones(n), x, _rng(9, 8), 7, 0.5)      # in place, with a residual
            _done()
            assert torch.equal(y, keep.to(dt) * 2) and torch.equal(x, keep.to(dt) * 2 + 1)
        for p in (1.0,):    # everything dropped
            x = torch.full((n,), float("nan"), dtype=dt, device="cuda")
            s2a.s2a_dropout_fwd(x, None, x, _rng(9, 8), 7, p)
            _done()
            assert bool((x == 0).all())


def test_dropout_in_place_and_into_the_residual():
    n = 5003
    x, r = _normal((n,), torch.bfloat16, "x"), _normal((n,), torch.bfloat16, "r")
    want = torch.empty_like(x)
    s2a.s2a_dropout_fwd(x, r, want, _rng(1, 2), 3, 0.3)
    for target in (0, 1):
        pair = [x.clone(), r.clone()]
        s2a.s2a_dropout_fwd(pair[0], pair[1], pair[target], _rng(1, 2), 3, 0.3)
        _done()
        assert torch.equal(pair[target], want) and torch.equal(pair[1 - target], (x, r)[1 - target])
    for p in (1.0,):
        pair = [x.clone(), r.clone()]
        s2a.s2a_dropout_fwd(pair[0], pair[1], pair[1], _rng(1, 2), 3, p)
        _done()
        assert torch.equal(pair[1], r)


def test_dropout_rate_and_independence_of_sites():
    n, p = 1 << 22, 0.3
    x = torch.ones(n, device="cuda")
    masks = []
    for site in (0, 1):
        y = torch.empty_like(x)
        s2a.s2a_dropout_fwd(x, None, y, _rng(11, 0), site, p)
        masks.append(y != 0)
    T = s2a.dropout_threshold(p)
    q = 1 - T / 65536
    for m in masks:     # six standard deviations of a binomial count
        assert abs(int(m.sum()) - n * q) <= 6 * math.sqrt(n * q * (1 - q))
    both = q * q
    assert abs(int((masks[0] & masks[1]).sum()) - n * both) <= 6 * math.sqrt(n * both * (1 - both))


def test_dropout_far_element():
    n = (1 << 32) + 24 + 5          # elements past 32 bits; 8.6 GB of bfloat16, in place
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    s2a.s2a_dropout_fwd(x, None, x, _rng(3, 4), 5, 0.5)
    _done()
    for first, m in ((0, 64), ((1 << 31) - 32, 64), ((1 << 32) - 32, 32 + 24 + 5)):
        want = _bits(m, 3, 4, 5, first) >= 32768
        assert np.array_equal(x[first:first + m].float().cpu().numpy(), want * 2.0)


# ------------------------------------------------------------------------------------------ relative position bias
def _map_of(buckets, tq, tk):
    b = buckets.long().cpu()
    if b.dim() == 2:
        return b
    return b[torch.arange(tk)[None, :] - torch.arange(tq)[:, None] + tq - 1]


def _check_bias(batch, heads, tq, tk, n, dtype, weights, form, outside=False):
    dt, wt = DT[dtype], DT[weights]
    key = (batch, heads, tq, tk, n, form)
    low, high = (-2, n + 2) if outside else (0, n)
    size = (tq, tk) if form == "map" else (tq + tk - 1,)
    buckets = torch.randint(low, high, size, generator=_gen("b", key), device="cuda").to(torch.int32)
    if outside:
        buckets.view(-1)[0] = -(1 << 31)
        buckets.view(-1)[-1] = (1 << 31) - 1
    table = _normal((n, heads), wt, "table", key)
    x = _normal((batch, heads, tq, tk), dt, "x", key)
    guard, y = _guarded((batch, heads, tq, tk), dt)
    s2a.s2a_relbias_fwd(x, table, buckets, y, batch, heads, tq, tk)
    _done()
    guard.check("y")
    where = _map_of(buckets, tq, tk).cuda()
    valid = (where >= 0) & (where < n)
    bias = torch.where(valid[..., None], table.double()[where.clamp(0, n - 1)], 0.0).permute(2, 0, 1)
    want = x.double() + bias
    _inside(y, want, (U + HALF[dt] * (1 + U)) * want.abs(), "bias forward")
    here = x.clone()
    s2a.s2a_relbias_fwd(here, table, buckets, here, batch, heads, tq, tk)
    _done()
    assert torch.equal(here, y)
    # whole-number gradients: every sum is exact in binary32, whatever its order
    g = torch.randint(-3, 4, (batch, heads, tq, tk), generator=_gen("g", key), device="cuda").to(dt)
    gt, grad = _guarded((n, heads), wt)
    gs, scratch = _guarded((s2a.relbias_scratch_bytes(batch, heads, tq, tk, n),), torch.uint8)
    s2a.s2a_relbias_bwd(g, buckets, grad, scratch, batch, heads, tq, tk)
    _done()
    gt.check("grad_table"), gs.check("scratch")
    flat = torch.where(valid, where, n).reshape(-1)
    exact = torch.zeros((n + 1, heads), dtype=torch.float64, device="cuda")
    exact.index_add_(0, flat, g.double().sum(0).reshape(heads, -1).t().contiguous())
    assert float(g.double().abs().sum()) < 2 ** 24
    assert torch.equal(grad, exact[:n].to(wt)), "the table's gradient of whole numbers must be exact"


BIAS_SHAPES = [(1, 1, 1, 1, 1), (2, 3, 1, 1, 4), (3, 2, 1, 7, 5), (2, 2, 7, 1, 8), (5, 3, 3, 5, 9), (9, 1, 7, 9, 64), (4, 5, 8, 8, 65),
               (17, 2, 13, 11, 33), (3, 12, 50, 50, 172), (2, 4, 49, 49, 172), (10, 3, 37, 41, 60), (2, 16, 1, 1025, 32),
               (40, 1, 1, 33, 32), (1, 2, 197, 197, 732), (11, 1, 65, 63, 7000), (1, 3, 90, 91, 9000), (3, 2, 33, 65, 20000),
               (1, 1, 200, 300, 32768), (2, 2, 129, 257, 16)]


@pytest.mark.parametrize("dtype,weights", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("form", ["map", "distance"])
@pytest.mark.parametrize("shape", BIAS_SHAPES)
def test_bias_forward_and_backward(shape, form, dtype, weights):
    _check_bias(*shape, dtype, weights, form)


@pytest.mark.parametrize("form", ["map", "distance"])
@pytest.mark.parametrize("shape", [(3, 2, 17, 19, 20), (2, 3, 31, 33, 100), (5, 1, 1, 40, 8)])
def test_bias_of_buckets_outside_the_table(shape, form):
    _check_bias(*shape, "f32", "f32", form, outside=True)


def test_bias_all_positions_in_one_bucket_and_in_none():
    for n in (3, 200):
        for u in (1, -1):
            buckets = torch.full((60, 61), u, dtype=torch.int32, device="cuda")
            g = torch.randint(-3, 4, (5, 2, 60, 61), generator=_gen("one"), device="cuda").bfloat16()
            grad = torch.full((n, 2), 9.0, device="cuda")
            scratch = torch.empty(s2a.relbias_scratch_bytes(5, 2, 60, 61, n), dtype=torch.uint8, device="cuda")
            s2a.s2a_relbias_bwd(g, buckets, grad, scratch, 5, 2, 60, 61)
            _done()
            want = torch.zeros((n, 2), device="cuda")
            if u >= 0:
                want[u] = g.float().sum((0, 2, 3))
            assert torch.equal(grad, want)


@pytest.mark.parametrize("n,form", [(32, "distance"), (700, "map")])
def test_bias_gradient_of_real_numbers(n, form):
    batch, heads, tq, tk = 6, 4, 150, 151
    buckets = torch.randint(0, n, (tq, tk) if form == "map" else (tq + tk - 1,), generator=_gen("b"), device="cuda").to(torch.int32)
    for dt in (torch.float32, torch.bfloat16):
        g = _normal((batch, heads, tq, tk), dt, "g")
        scratch = torch.empty(s2a.relbias_scratch_bytes(batch, heads, tq, tk, n), dtype=torch.uint8, device="cuda")
        outs = []
        for _ in range(3):
            grad = torch.empty((n, heads), device="cuda")
            scratch.fill_(0xFF)
            s2a.s2a_relbias_bwd(g, buckets, grad, scratch, batch, heads, tq, tk)
            outs.append(grad)
        _done()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]), "repeated calls must give the same bits"
        where = _map_of(buckets, tq, tk).cuda().reshape(-1)
        zero = torch.zeros((n, heads), dtype=torch.float64, device="cuda")
        flat = g.double().sum(0).reshape(heads, -1).t().contiguous()
        size = g.double().abs().sum(0).reshape(heads, -1).t().contiguous()
        want, mass = zero.index_add(0, where, flat), zero.index_add(0, where, size)
        _inside(outs[0], want, (batch + 2048) * U * mass, "grad_table")


def test_bias_keeps_masked_scores():
    batch, heads, t, n = 2, 3, 21, 32
    x = _normal((batch, heads, t, t), torch.bfloat16, "x")
    x[:, :, 4] = float("-inf")                                   # a row that the mask leaves empty
    x[:, :, :, 9:] = float("-inf")
    x[0, 0, 0, 0] = float("nan")
    x[0, 0, 0, 1] = float("inf")
    x[0, 0, 1, 0] = torch.finfo(torch.bfloat16).min
    table = _normal((n, heads), torch.float32, "t")
    lut = s2a.log_buckets(1 - t, 2 * t - 1, n, 64, True).cuda()
    y = torch.empty_like(x)
    s2a.s2a_relbias_fwd(x, table, lut, y, batch, heads, t, t)
    _done()
    where = _map_of(lut, t, t).cuda()
    want = (x.float() + table[where].permute(2, 0, 1)).bfloat16()
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y.nan_to_num(1.0), want.nan_to_num(1.0))


def test_bias_empty_shapes_zero_the_gradient():
    lut = torch.zeros(8, dtype=torch.int32, device="cuda")
    grad = torch.full((5, 3), 9.0, dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(16, dtype=torch.uint8, device="cuda")
    s2a.s2a_relbias_bwd(torch.empty((0, 3, 4, 5), device="cuda"), lut, grad, scratch, 0, 3, 4, 5)
    _done()
    assert bool((grad == 0).all())


def test_bias_one_new_token_reads_a_window_of_a_long_vector():
    """A growing cache: the buckets of all distances are laid out once, and step t takes its window."""
    longest, n, heads, batch = 300, 32, 4, 3
    lut = s2a.log_buckets(1 - longest, longest, n, 128, False).cuda()     # distances 1 - longest .. 0
    table = _normal((n, heads), torch.bfloat16, "t")
    for length in (1, 2, 9, 64, 299, 300):
        x = _normal((batch, heads, 1, length), torch.float32, "x", length)
        y = torch.empty_like(x)
        s2a.s2a_relbias_fwd(x, table, lut[longest - length:], y, batch, heads, 1, length)
        _done()
        want = x + table.float()[lut[longest - length:].long()].t()[None, :, None, :]
        assert torch.equal(y, want)


def test_bias_slabs_beyond_32_bit_offsets():
    batch, heads, tq, tk, n = 3, 1, 1 << 15, (1 << 16) + 1, 16            # 2.1e9 positions a slab, 12.9 GB of bfloat16
    x = torch.ones((batch, heads, tq, tk), dtype=torch.bfloat16, device="cuda")
    d = torch.arange(tq + tk - 1, device="cuda")
    lut = (d % n).to(torch.int32)
    table = torch.arange(n, dtype=torch.float32, device="cuda")[:, None].contiguous()
    s2a.s2a_relbias_fwd(x, table, lut, x, batch, heads, tq, tk)
    _done()
    for b, q in ((0, 0), (1, tq - 1), (2, 5), (2, tq - 1)):
        want = 1 + table[lut[tq - 1 - q:tq - 1 - q + tk].long(), 0]
        assert torch.equal(x[b, 0, q].float(), want)
    # gradients that are one on the last sample's last row and zero elsewhere
    x.zero_()
    x[2, 0, tq - 1] = 1
    grad = torch.empty((n, 1), device="cuda")
    scratch = torch.empty(s2a.relbias_scratch_bytes(batch, heads, tq, tk, n), dtype=torch.uint8, device="cuda")
    s2a.s2a_relbias_bwd(x, lut, grad, scratch, batch, heads, tq, tk)
    _done()
    assert torch.equal(grad[:, 0], torch.bincount(lut[:tk].long(), minlength=n).float())


# ------------------------------------------------------------------------------------------ streams, graphs, arguments
def _norm_problem(rows=700, L=768):
    x, g = _normal((rows, L), torch.bfloat16, "x", rows), _normal((rows, L), torch.bfloat16, "g", rows)
    gamma = _normal((L,), torch.float32, "gamma")
    return x, g, gamma


def test_calls_on_two_streams_with_a_scratch_each():
    x, g, gamma = _norm_problem()
    L = x.shape[1]
    _, stats = _norm_fwd(x, gamma, gamma, L)
    want = _check_norm_bwd(g, x, gamma, stats, L)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(t) for t in want] for _ in streams]
    scratch = [torch.empty(s2a.layernorm_scratch_bytes(*x.shape), dtype=torch.uint8, device="cuda") for _ in streams]
    for _ in range(20):
        for s, o, w in zip(streams, outs, scratch):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                s2a.s2a_layernorm_bwd(g, x, gamma, stats, o[0], o[1], o[2], w, L)
    _done()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, want))


def test_captured_step_replays_and_draws_new_masks():
    x, g, gamma = _norm_problem(64)
    L = x.shape[1]
    rng = _rng(5, 100)
    y, stats, dropped, gin = torch.empty_like(x), torch.empty((64, 2), device="cuda"), torch.empty_like(x), torch.empty_like(x)
    dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(gamma)
    scratch = torch.empty(s2a.layernorm_scratch_bytes(64, L), dtype=torch.uint8, device="cuda")

    def step():
        s2a.s2a_layernorm_fwd(x, gamma, gamma, y, stats, L, 1e-6)
        s2a.s2a_dropout_fwd(y, x, dropped, rng, 1, 0.2)
        s2a.s2a_dropout_bwd(g, gin, rng, 1, 0.2)
        s2a.s2a_layernorm_bwd(gin, x, gamma, stats, gin, dgamma, dbeta, scratch, L)

    outs = (y, stats, dropped, gin, dgamma, dbeta)
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.synchronize()
    seen = []
    for k in range(3):
        rng[1] = 100 + 10 * k
        x.copy_(_normal(x.shape, x.dtype, "new", k))
        for t in outs:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        for t in outs:
            t.fill_(7)
        step()
        _done()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs))
        seen.append(replayed[2] - x.to(replayed[2].dtype) == 0)
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_binding_refusals():
    x = torch.zeros((4, 64), device="cuda")
    w, st = torch.ones(64, device="cuda"), torch.empty((4, 2), device="cuda")
    E = s2a.S2AError
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w, w, x.bfloat16(), st, 64, 1e-6)            # y of another dtype
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w, w, x[:3], st, 64, 1e-6)                   # y too small
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w[:60], w, x, st, 64, 1e-6)                  # gamma of another length
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w, w.bfloat16(), x, st, 64, 1e-6)            # weights of two dtypes
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w, w, x, st.bfloat16(), 64, 1e-6)
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x.half(), w, w, x.half(), st, 64, 1e-6)         # float16
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w, w, x, st, 60, 1e-6)                       # not whole rows
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x.t(), w[:4], w[:4], torch.empty((64, 4), device="cuda"), None, 4, 1e-6)
    with pytest.raises(E):
        s2a.s2a_layernorm_fwd(x, w, w, x, st, 64, -1.0)
    with pytest.raises(E, match="scratch"):
        s2a.s2a_layernorm_bwd(x, x, w, st, torch.empty_like(x), w.clone(), None, None, 64)
    with pytest.raises(E, match="scratch"):
        s2a.s2a_layernorm_bwd(x, x, w, st, torch.empty_like(x), w.clone(), None, torch.empty(8, dtype=torch.uint8, device="cuda"), 64)
    with pytest.raises(E, match="stats"):
        s2a.s2a_layernorm_bwd(x, x, w, None, torch.empty_like(x), None, None, None, 64)
    with pytest.raises(E):
        s2a.s2a_dropout_fwd(x, None, x, torch.zeros(2, device="cuda"), 0, 0.5)
    with pytest.raises(E):
        s2a.s2a_dropout_fwd(x, None, x, _rng(0, 0).cpu(), 0, 0.5)             # another device
    with pytest.raises(E):
        s2a.s2a_dropout_fwd(x, x[:2], x, _rng(0, 0), 0, 0.5)
    with pytest.raises(E):
        s2a.s2a_dropout_fwd(x[:, 1:], None, x[:, 1:], _rng(0, 0), 0, 0.5)     # not contiguous
    with pytest.raises(E):
        s2a.s2a_dropout_fwd(x.view(-1)[1:], None, x.view(-1)[1:], _rng(0, 0), 0, 0.5)   # off the 16-byte grid
    with pytest.raises(E):
        s2a.s2a_dropout_fwd(x, None, x, _rng(0, 0), 0, 1.5)
    lut, table = torch.zeros(7, dtype=torch.int32, device="cuda"), torch.zeros((4, 4), device="cuda")
    s = torch.zeros((4, 4, 2, 6), device="cuda")
    s2a.s2a_relbias_fwd(s, table, lut, s, 4, 4, 2, 6)
    with pytest.raises(E):
        s2a.s2a_relbias_fwd(s, table, lut[:6], s, 4, 4, 2, 6)                 # the vector is too short
    with pytest.raises(E):
        s2a.s2a_relbias_fwd(s, table, lut.long(), s, 4, 4, 2, 6)
    with pytest.raises(E):
        s2a.s2a_relbias_fwd(s, table[:, :3], lut, s, 4, 4, 2, 6)
    with pytest.raises(E):
        s2a.s2a_relbias_fwd(s, table, lut, s, 4, 4, 3, 6)
    with pytest.raises(E, match="scratch"):
        s2a.s2a_relbias_bwd(s, lut, table, torch.empty(4, dtype=torch.uint8, device="cuda"), 4, 4, 2, 6)
    _done()


# ------------------------------------------------------------------------------------------ a block's layers together
def test_layers_of_a_block_together():
    """norm -> scores -> bias -> softmax with its stash -> dropout -> values -> dropout + residual -> norm -> GELU with its
    stash -> dropout + residual and all the way back, with torch's matrix products between.  Each new layer's output is
    checked against 64 bits on the inputs that the kernels before it really gave."""
    B, H, T, d, hidden, p = 3, 4, 50, 32, 256, 0.1
    Cn, dt = H * d, torch.bfloat16
    n_buckets = 32
    rng = _rng(21, 0)
    h = _normal((B * T, Cn), dt, "h")
    ones = lambda k: (_normal((Cn,), torch.float32, "w", k) * 0.1 + 1)
    g1, b1, g2, b2 = ones(0), ones(1) - 1, ones(2), ones(3) - 1
    wqkv, wo = _normal((Cn, 3 * Cn), dt, "wqkv", scale=Cn ** -0.5), _normal((Cn, Cn), dt, "wo", scale=Cn ** -0.5)
    w1, w2 = _normal((Cn, hidden), dt, "w1", scale=Cn ** -0.5), _normal((hidden, Cn), dt, "w2", scale=hidden ** -0.5)
    lut = s2a.log_buckets(1 - T, 2 * T - 1, n_buckets, 64, True).cuda()
    table = _normal((n_buckets, H), torch.float32, "table")
    n = B * T

    def drop(x, r, site):
        y = torch.empty_like(x)
        s2a.s2a_dropout_fwd(x, r, y, rng, site, p)
        keep = torch.from_numpy(_bits(x.numel(), 21, 0, site) >= s2a.dropout_threshold(p)).cuda().view(x.shape)
        part = torch.where(keep, x.double(), 0.0) * (65536 / (65536 - s2a.dropout_threshold(p)))
        want = part if r is None else part + r.double()
        _inside(y, want, 2 * U * part.abs() + (U + HALF[dt]) * want.abs() * (1 + 2 * U), "dropout %d" % site)
        return y

    # forward
    n1, st1 = _check_norm_fwd(h, g1, b1, Cn)
    qkv = (n1 @ wqkv).view(B, T, 3, H, d).permute(2, 0, 3, 1, 4)
    q, k, v = (t.contiguous() for t in qkv)
    scores = (q @ k.transpose(-1, -2)) * d ** -0.5
    scores = scores.contiguous()
    biased = torch.empty_like(scores)
    s2a.s2a_relbias_fwd(scores, table, lut, biased, B, H, T, T)
    where = _map_of(lut, T, T).cuda()
    want = scores.double() + table.double()[where].permute(2, 0, 1)
    _inside(biased, want, (U + HALF[dt] * (1 + U)) * want.abs(), "bias")
    prob = torch.empty_like(biased)
    codes, meta = s2a.alloc_stash(prob.numel(), T, prob.device)
    s2a.s2a_softmax_fwd(biased, prob, codes, meta, T)
    att = drop(prob, None, 0)
    mixed = (att @ v).permute(0, 2, 1, 3).reshape(n, Cn)
    proj = mixed @ wo
    h1 = drop(proj, h, 1)
    n2, st2 = _check_norm_fwd(h1, g2, b2, Cn)
    up = n2 @ w1
    act = torch.empty_like(up)
    gcodes, gmeta = s2a.alloc_stash(up.numel(), hidden, up.device)
    s2a.s2a_gelu_fwd(up, act, gcodes, gmeta, hidden)
    down = act @ w2
    h2 = drop(down, h1, 2)
    # backward
    def undrop(g, site):
        out = torch.empty_like(g)
        s2a.s2a_dropout_bwd(g, out, rng, site, p)
        assert torch.equal(out, drop(g, None, site))
        return out

    gh2 = _normal((n, Cn), dt, "gh2", scale=0.1)
    gact = undrop(gh2, 2) @ w2.t()
    gup = torch.empty_like(gact)
    s2a.s2a_gelu_bwd(gact, gcodes, gmeta, gup, hidden)
    gn2 = gup @ w1.t()
    gin2, dg2, db2 = _check_norm_bwd(gn2, h1, g2, st2, Cn)
    gh1 = gh2 + gin2
    gmixed = (undrop(gh1, 1) @ wo.t()).view(B, T, H, d).permute(0, 2, 1, 3)
    gprob = undrop((gmixed @ v.transpose(-1, -2)).contiguous(), 0)
    gscores = torch.empty_like(gprob)
    s2a.s2a_softmax_bwd(gprob, codes, meta, gscores, T)
    gtable = torch.empty_like(table)
    scratch = torch.empty(s2a.relbias_scratch_bytes(B, H, T, T, n_buckets), dtype=torch.uint8, device="cuda")
    s2a.s2a_relbias_bwd(gscores, lut, gtable, scratch, B, H, T, T)
    zero = torch.zeros((n_buckets, H), dtype=torch.float64, device="cuda")
    pick = lambda t: t.sum(0).reshape(H, -1).t().contiguous()
    exact = zero.index_add(0, where.reshape(-1), pick(gscores.double()))
    mass = zero.index_add(0, where.reshape(-1), pick(gscores.double().abs()))
    _inside(gtable, exact, (B + 2048) * U * mass, "grad_table")
    gs = gscores * d ** -0.5
    gq, gk = gs @ k, gs.transpose(-1, -2) @ q
    gv = att.transpose(-1, -2) @ gmixed
    gqkv = torch.stack([gq, gk, gv]).permute(1, 3, 0, 2, 4).reshape(n, 3 * Cn)
    gn1 = gqkv @ wqkv.t()
    gin1, dg1, db1 = _check_norm_bwd(gn1, h, g1, st1, Cn)
    gh = gh1 + gin1
    _done()
    for t in (h2, gh, gtable, dg1, db1, dg2, db2):
        assert bool(torch.isfinite(t).all()) and float(t.abs().max()) > 0
