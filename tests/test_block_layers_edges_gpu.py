"""Layer norm, dropout and the relative position bias where their kernels change path: seeded walks over shapes, strides and
alignments, non-finite neighbours of rows that share a vector, broadcast and interleaved rows, the first call of a process
under stream capture, and calls on tensors' slices.  Tolerances are those of test_block_layers_gpu.py."""
import os
import random
import subprocess
import sys

import pytest
import torch

import test_block_layers_gpu as base
from paper_2503_08154_b200 import binding as s2a

pytestmark = pytest.mark.gpu

U, HALF = base.U, base.HALF
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _place(rows, L, rng, dtype, *key):
    """Rows of L elements in a buffer of their own, at a random offset and stride, and the mask of what is not theirs."""
    stride = L + rng.choice([0, 0, 1, 3, 8, 16])
    offset = rng.choice([0, 0, 1, 2, 5, 8])
    buf = base._normal((rows * stride + offset + 16,), dtype, *key)
    view = buf[offset:offset + rows * stride].view(rows, stride)[:, :L]
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[offset:offset + rows * stride].view(rows, stride)[:, :L] = False
    return buf, view, rest


@pytest.mark.parametrize("seed", range(40))
def test_norm_walk_over_shapes_strides_and_alignments(seed):
    rng = random.Random(seed)
    dt = rng.choice([torch.float32, torch.bfloat16])
    wt = rng.choice([torch.float32, torch.bfloat16])
    L = rng.choice([rng.randint(1, 70), rng.randint(60, 300), rng.randint(250, 1100), rng.randint(1000, 3000), rng.choice([64, 512, 1024, 4096]),
                    rng.randint(8000, 17000)])
    rows = rng.randint(1, max(2, min(3000, 400_000 // L)))
    _, x, _ = _place(rows, L, rng, dt, "x", seed)
    _, g, _ = _place(rows, L, rng, dt, "g", seed)
    ybuf, y, rest = _place(rows, L, rng, dt, "y", seed)
    before = ybuf[rest].clone()
    # the weights' own alignment may be anything too
    gamma = base._normal((L + 3,), wt, "gamma", seed)[rng.choice([0, 1, 3]):][:L]
    beta = base._normal((L + 3,), wt, "beta", seed)[rng.choice([0, 1, 3]):][:L]
    stats = torch.empty((rows, 2), device="cuda")
    s2a.s2a_layernorm_fwd(x, gamma, beta, y, stats, L, 1e-5)
    base._done()
    want, mean, rstd, tol, tm, tr = base._norm_exact(x, gamma, beta, 1e-5)
    base._inside(stats[:, :1], mean, tm + U * mean.abs(), "mean")
    base._inside(stats[:, 1:], rstd, tr, "rstd")
    base._inside(y, want, tol + HALF[dt] * (want.abs() + tol), "y")
    assert torch.equal(ybuf[rest], before), "elements outside the rows were written"
    dgamma, dbeta = (torch.empty(L + 1, dtype=wt, device="cuda")[1:] for _ in range(2))
    scratch = torch.empty(s2a.layernorm_scratch_bytes(rows, L), dtype=torch.uint8, device="cuda").fill_(0xFF)
    s2a.s2a_layernorm_bwd(g, x, gamma, stats, y, dgamma, dbeta, scratch, L)
    base._done()
    dx, dg, db, tol, tg, tb = base._norm_bwd_tolerance(g, x, gamma, stats)
    base._inside(y, dx, tol + HALF[dt] * (dx.abs() + tol), "grad_in")
    base._inside(dgamma, dg, tg + HALF[wt] * (dg.abs() + tg), "grad_gamma")
    base._inside(dbeta, db, tb + HALF[wt] * (db.abs() + tb), "grad_beta")
    assert torch.equal(ybuf[rest], before)


@pytest.mark.parametrize("L", [63, 197, 1025, 2049])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_neighbouring_rows_that_share_a_vector_do_not_leak(L, dtype):
    dt, rows = base.DT[dtype], 24
    x = base._normal((rows, L), dt, "x", L)
    g = base._normal((rows, L), dt, "g", L)
    bad = torch.zeros(rows, dtype=torch.bool)
    bad[1::3] = True
    for poison in (float("nan"), float("inf"), torch.finfo(dt).max):
        xp, gp = x.clone(), g.clone()
        xp[bad.cuda()] = poison
        gp[bad.cuda()] = poison
        y, stats = base._norm_fwd(x, None, None, L)
        yp, sp = base._norm_fwd(xp, None, None, L)
        good = (~bad).cuda()
        assert torch.equal(yp[good], y[good]) and torch.equal(sp[good], stats[good])
        gin, ginp = torch.empty_like(x), torch.empty_like(x)
        s2a.s2a_layernorm_bwd(g, x, None, stats, gin, None, None, None, L)
        s2a.s2a_layernorm_bwd(gp, xp, None, torch.where(good[:, None], stats, sp), ginp, None, None, None, L)
        base._done()
        assert torch.equal(ginp[good], gin[good])


def test_norm_broadcast_input_and_interleaved_rows():
    L, rows = 200, 37
    one = base._normal((1, L), torch.bfloat16, "one")
    gamma = base._normal((L,), torch.float32, "gamma")
    y, stats = base._norm_fwd(one, gamma, gamma, L)
    many = torch.empty((rows, L), dtype=torch.bfloat16, device="cuda")
    st = torch.empty((rows, 2), device="cuda")
    s2a.s2a_layernorm_fwd(one.expand(rows, L), gamma, gamma, many, st, L, 1e-6)
    base._done()
    assert torch.equal(many, y.expand(rows, L)) and torch.equal(st, stats.expand(rows, 2))
    # x and y as the two halves of every row of one buffer
    for half in (200, 201):
        buf = base._normal((rows, 2 * half), torch.bfloat16, "buf", half)
        x = buf[:, :half].clone()
        want, _ = base._norm_fwd(x, None, None, half)
        s2a.s2a_layernorm_fwd(buf[:, :half], None, None, buf[:, half:], st, half, 1e-6)
        base._done()
        assert torch.equal(buf[:, :half], x)
        got, exact = buf[:, half:], base._norm_exact(x, None, None, 1e-6)
        base._inside(got, exact[0], exact[3] + HALF[torch.bfloat16] * (exact[0].abs() + exact[3]), "interleaved")
    with pytest.raises(s2a.S2AError, match="OVERLAP"):
        s2a.s2a_layernorm_fwd(buf[:, :half], None, None, buf[:, half - 1:-1], st, half, 1e-6)


@pytest.mark.parametrize("seed", range(60))
def test_bias_walk_over_shapes(seed):
    rng = random.Random(1000 + seed)
    form = rng.choice(["map", "distance"])
    tq = rng.choice([1, 1, rng.randint(2, 20), rng.randint(15, 80), rng.randint(100, 400)])
    tk = rng.choice([1, rng.randint(2, 20), rng.randint(15, 80), rng.randint(60, 700)])
    heads = rng.choice([1, 2, 3, 7, 8, 12, 16])
    batch = rng.randint(1, max(1, min(140, 1_500_000 // (tq * tk * heads))))
    n = rng.choice([1, 2, 8, 32, 64, 300, 732, 3000])
    dtype, weights = rng.choice([("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
    base._check_bias(batch, heads, tq, tk, n, dtype, weights, form, outside=n > 1 and rng.random() < 0.3)


@pytest.mark.parametrize("form,tq,tk", [("map", 37, 41), ("distance", 37, 41), ("distance", 3, 13), ("distance", 1, 101)])
def test_bias_gradient_keeps_a_nan_in_its_bucket(form, tq, tk):
    batch, heads, n = 5, 3, 40
    size = (tq, tk) if form == "map" else (tq + tk - 1,)
    buckets = torch.randint(0, n, size, generator=base._gen("b", form, tq), device="cuda").to(torch.int32)
    where = base._map_of(buckets, tq, tk)
    for dt in (torch.float32, torch.bfloat16):
        clean = torch.randint(-3, 4, (batch, heads, tq, tk), generator=base._gen("g"), device="cuda").to(dt)
        scratch = torch.empty(s2a.relbias_scratch_bytes(batch, heads, tq, tk, n), dtype=torch.uint8, device="cuda")
        want = torch.empty((n, heads), device="cuda")
        s2a.s2a_relbias_bwd(clean, buckets, want, scratch, batch, heads, tq, tk)
        for b, h, q, k in ((0, 0, 0, 0), (1, 2, tq - 1, tk - 1), (batch - 1, heads - 1, tq - 1, tk - 1), (2, 1, tq // 2, 0), (3, 0, 0, tk - 1)):
            g = clean.clone()
            g[b, h, q, k] = float("nan")
            grad = torch.empty((n, heads), device="cuda")
            s2a.s2a_relbias_bwd(g, buckets, grad, scratch, batch, heads, tq, tk)
            base._done()
            expect = want.clone()
            expect[int(where[q, k]), h] = float("nan")
            assert torch.equal(torch.isnan(grad), torch.isnan(expect))
            assert torch.equal(grad.nan_to_num(7.0), expect.nan_to_num(7.0))


def test_bias_gradient_is_the_forward_pass_transposed():
    """<bias(table), g> = <table, grad_table> for every table and gradient: both sides are sums of whole numbers here, so exact."""
    batch, heads, tq, tk, n = 4, 3, 45, 51, 32
    lut = s2a.log_buckets(1 - tk, tq + tk - 1, n, 40, True).cuda()
    table = torch.randint(-9, 10, (n, heads), generator=base._gen("t"), device="cuda").float()
    g = torch.randint(-3, 4, (batch, heads, tq, tk), generator=base._gen("g"), device="cuda").float()
    y = torch.empty_like(g)
    s2a.s2a_relbias_fwd(torch.zeros_like(g), table, lut, y, batch, heads, tq, tk)
    grad = torch.empty_like(table)
    scratch = torch.empty(s2a.relbias_scratch_bytes(batch, heads, tq, tk, n), dtype=torch.uint8, device="cuda")
    s2a.s2a_relbias_bwd(g, lut, grad, scratch, batch, heads, tq, tk)
    base._done()
    assert float((y.double() * g.double()).sum()) == float((table.double() * grad.double()).sum())


def test_dropout_of_slices_repeats_the_whole_tensors_mask():
    # element e of a call has a mask of its own, wherever the call ends
    n = 4096
    x = torch.ones(n, device="cuda")
    whole = torch.empty_like(x)
    s2a.s2a_dropout_fwd(x, None, whole, base._rng(9, 1), 2, 0.4)
    for m in (1, 7, 100, 1031):
        part = torch.zeros(m, device="cuda")
        s2a.s2a_dropout_fwd(x[:m], None, part, base._rng(9, 1), 2, 0.4)
        base._done()
        assert torch.equal(part, whole[:m])
        half = torch.zeros(m, dtype=torch.bfloat16, device="cuda")
        s2a.s2a_dropout_fwd(x[:m].bfloat16(), None, half, base._rng(9, 1), 2, 0.4)
        base._done()
        assert torch.equal(half != 0, part != 0), "the mask does not depend on the type"


CAPTURE = """
import sys
sys.path.insert(0, %r)
import torch
from paper_2503_08154_b200 import binding as s2a
x = torch.randn(300, 1025, device="cuda"); w = torch.randn(1025, device="cuda"); st = torch.empty(300, 2, device="cuda")
y, gx, gw, gb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
sc = torch.empty(s2a.layernorm_scratch_bytes(300, 1025), dtype=torch.uint8, device="cuda")
rng = torch.tensor([1, 2], device="cuda")
s = torch.randn(4, 3, 40, 40, device="cuda"); t = torch.randn(700, 3, device="cuda"); gt = torch.empty_like(t)
m = torch.randint(0, 700, (40, 40), device="cuda").to(torch.int32); sb = torch.empty_like(s)
sc2 = torch.empty(s2a.relbias_scratch_bytes(4, 3, 40, 40, 700), dtype=torch.uint8, device="cuda")
def step():
    s2a.s2a_layernorm_fwd(x, w, w, y, st, 1025, 1e-6)
    s2a.s2a_dropout_fwd(y, x, y, rng, 3, 0.5)
    s2a.s2a_layernorm_bwd(y, x, w, st, gx, gw, gb, sc, 1025)
    s2a.s2a_relbias_fwd(s, t, m, sb, 4, 3, 40, 40)
    s2a.s2a_relbias_bwd(sb, m, gt, sc2, 4, 3, 40, 40)
torch.cuda.synchronize()
stream = torch.cuda.Stream()
with torch.cuda.stream(stream):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):   # the library's first calls in this process
        step()
for o in (y, gx, gw, gb, sb, gt):
    o.fill_(7)
torch.cuda.synchronize()
graph.replay()
torch.cuda.synchronize()
got = [o.clone() for o in (y, gx, gw, gb, sb, gt)]
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (y, gx, gw, gb, sb, gt)))
print("same")
"""


def test_first_calls_of_a_process_may_be_captured():
    r = subprocess.run([sys.executable, "-c", CAPTURE % ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


# Few samples under a map, or of one query row, are taken element by element: a table that fits beside them in shared memory, ones that are
# too large or larger than what a CTA looks up, several rounds of a CTA, ragged ends.
@pytest.mark.parametrize("batch,heads,tq,tk,n", [(1, 1, 1, 1, 1), (1, 2, 70, 71, 20), (2, 5, 33, 31, 2000), (4, 3, 65, 67, 5000), (2, 1, 97, 131, 12289),
                                                 (1, 300, 130, 150, 12288), (3, 16, 1, 9001, 32), (4, 12, 197, 197, 732), (2, 7, 130, 257, 32768)])
@pytest.mark.parametrize("dtype,weights", [("f32", "bf16"), ("bf16", "f32")])
def test_bias_of_few_samples(batch, heads, tq, tk, n, dtype, weights):
    for form in ("map", "distance") if tq == 1 else ("map",):
        base._check_bias(batch, heads, tq, tk, n, dtype, weights, form, outside=n > 1)


@pytest.mark.parametrize("tq,tk,n", [(50, 50, 172), (37, 129, 40), (1, 4097, 32)])
def test_bias_of_a_sample_does_not_depend_on_the_others(tq, tk, n):
    heads = 3
    x = base._normal((9, heads, tq, tk), torch.bfloat16, "x")
    x[:, :, :, 5::11] = float("-inf")
    table = base._normal((n, heads), torch.float32, "t")
    buckets = torch.randint(0, n, (tq, tk), generator=base._gen("b"), device="cuda").to(torch.int32)
    whole = torch.empty_like(x)
    s2a.s2a_relbias_fwd(x, table, buckets, whole, 9, heads, tq, tk)
    for batch in range(1, 9):
        part, y = x[:batch].contiguous(), torch.empty_like(x[:batch])
        s2a.s2a_relbias_fwd(part, table, buckets, y, batch, heads, tq, tk)
        base._done()
        assert torch.equal(y, whole[:batch])


@pytest.mark.parametrize("batch,n", [(1, 32), (2, 700), (4, 9000)])
def test_bias_gradient_of_few_samples_and_real_numbers(batch, n):
    heads, tq, tk = 4, 150, 151
    buckets = torch.randint(-1, n, (tq, tk), generator=base._gen("b", n), device="cuda").to(torch.int32)
    buckets[3] = 2                                  # runs of one bucket
    buckets[5, ::2] = 4                             # and one bucket met again within a warp
    for dt in (torch.float32, torch.bfloat16):
        g = base._normal((batch, heads, tq, tk), dt, "g")
        g[:, :, buckets == -1] = float("nan")       # what has no bucket leaves no trace
        scratch = torch.empty(s2a.relbias_scratch_bytes(batch, heads, tq, tk, n), dtype=torch.uint8, device="cuda")
        outs = []
        for _ in range(3):
            grad = torch.empty((n, heads), device="cuda")
            scratch.fill_(0xFF)
            s2a.s2a_relbias_bwd(g, buckets, grad, scratch, batch, heads, tq, tk)
            outs.append(grad)
        base._done()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]), "repeated calls must give the same bits"
        where = buckets.long().reshape(-1)
        flat = g.double().sum(0).reshape(heads, -1).t()[where >= 0]
        size = g.double().abs().sum(0).reshape(heads, -1).t()[where >= 0]
        zero = torch.zeros((n, heads), dtype=torch.float64, device="cuda")
        want, mass = zero.index_add(0, where[where >= 0], flat), zero.index_add(0, where[where >= 0], size)
        # a sum of at most batch * count terms, in any order: (terms - 1) roundings each
        terms = batch * int(torch.bincount(where[where >= 0]).max())
        base._inside(outs[0], want, terms * U * mass, "grad_table")
