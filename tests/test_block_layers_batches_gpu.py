"""The relative position bias on both sides of the batch sizes at which its kernels change (4 samples forward, 8 backward, where there is one
query row or a map), and with few and many query rows by distance.

A sum of n terms, in any order, is off by at most n u sum|terms|, u = 2^-24."""
import subprocess
import sys

import pytest
import torch

import test_block_layers_edges_gpu as edges
import test_block_layers_gpu as base
from paper_2503_08154_b200 import binding as s2a

pytestmark = pytest.mark.gpu

U = base.U
BATCHES = [1, 4, 5, 8, 9, 17]
FORMS = [("map", 37, 41), ("map", 1, 101), ("distance", 1, 101), ("distance", 3, 13), ("distance", 40, 41)]


def _buckets(form, tq, tk, n, low=0):
    size = (tq, tk) if form == "map" else (tq + tk - 1,)
    return torch.randint(low, n, size, generator=base._gen("b", form, tq, n), device="cuda").to(torch.int32)


def _grad(g, buckets, n, dtype=torch.float32):
    batch, heads, tq, tk = g.shape
    guard, grad = base._guarded((n, heads), dtype)
    scratch = torch.empty(s2a.relbias_scratch_bytes(batch, heads, tq, tk, n), dtype=torch.uint8, device="cuda").fill_(0xFF)
    s2a.s2a_relbias_bwd(g, buckets, grad, scratch, batch, heads, tq, tk)
    base._done()
    guard.check("grad_table")
    return grad


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("form,tq,tk", FORMS)
def test_bias_gradient_of_real_numbers_is_near_and_repeats(form, tq, tk, batch):
    heads = 3
    for n in (5, 300):
        buckets = _buckets(form, tq, tk, n, low=-1)
        where = base._map_of(buckets, tq, tk).cuda().reshape(-1)
        held = where >= 0
        terms = batch * int(torch.bincount(where[held], minlength=1).max())
        for dt in (torch.float32, torch.bfloat16):
            g = base._normal((batch, heads, tq, tk), dt, "g", batch)
            g[:, :, ~held.reshape(tq, tk)] = float("nan")            # what has no bucket leaves no trace
            outs = [_grad(g, buckets, n) for _ in range(3)]
            assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]), "repeated calls must give the same bits"
            pick = lambda t: t.double().sum(0).reshape(heads, -1).t()[held]
            zero = torch.zeros((n, heads), dtype=torch.float64, device="cuda")
            want, mass = zero.index_add(0, where[held], pick(g)), zero.index_add(0, where[held], pick(g.abs()))
            base._inside(outs[0], want, terms * U * mass, "grad_table")


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("form,tq,tk", FORMS)
def test_bias_gradient_keeps_a_nan_in_its_bucket_in_every_batch(form, tq, tk, batch):
    heads, n = 3, 40
    buckets = _buckets(form, tq, tk, n)
    where = base._map_of(buckets, tq, tk)
    for dt in (torch.float32, torch.bfloat16):
        clean = torch.randint(-3, 4, (batch, heads, tq, tk), generator=base._gen("g"), device="cuda").to(dt)
        want = _grad(clean, buckets, n)
        last = batch - 1
        for b, h, q, k in ((0, 0, 0, 0), (last, heads - 1, tq - 1, tk - 1), (batch // 2, 1, tq // 2, 0), (last, 0, 0, tk - 1), (0, 2, tq - 1, 0)):
            for bad in (float("nan"), float("inf")):
                g = clean.clone()
                g[b, h, q, k] = bad
                expect = want.clone()
                expect[int(where[q, k]), h] = bad
                got = _grad(g, buckets, n)
                assert torch.equal(torch.isnan(got), torch.isnan(expect))
                assert torch.equal(got.nan_to_num(7.0), expect.nan_to_num(7.0))


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("form,tq,tk", FORMS)
def test_bias_with_all_positions_in_one_bucket_in_none_and_outside(form, tq, tk, batch):
    heads = 2
    size = (tq, tk) if form == "map" else (tq + tk - 1,)
    g = torch.randint(-3, 4, (batch, heads, tq, tk), generator=base._gen("one", batch), device="cuda").bfloat16()
    for n in (3, 200):
        for u in (1, -1, n, -(1 << 31), (1 << 31) - 1):
            buckets = torch.full(size, u, dtype=torch.int32, device="cuda")
            want = torch.zeros((n, heads), device="cuda")
            if u == 1:
                want[u] = g.float().sum((0, 2, 3))
            assert torch.equal(_grad(g, buckets, n), want)
            table, y = torch.full((n, heads), 2.0, device="cuda"), torch.empty_like(g)
            s2a.s2a_relbias_fwd(g, table, buckets, y, batch, heads, tq, tk)
            base._done()
            assert torch.equal(y, g + 2 if u == 1 else g)


@pytest.mark.parametrize("batch", [3, 4, 5, 8, 9, 16, 17])
@pytest.mark.parametrize("form,tq,tk,n", [("map", 17, 19, 20), ("map", 31, 33, 2000), ("distance", 1, 40, 8), ("distance", 17, 19, 20), ("map", 130, 131, 9000)])
def test_bias_of_buckets_outside_the_table_in_every_batch(form, tq, tk, n, batch):
    for dtype, weights in (("f32", "bf16"), ("bf16", "f32")):
        base._check_bias(batch, 2, tq, tk, n, dtype, weights, form, outside=True)


@pytest.mark.parametrize("batch", [4, 8, 9, 17])
def test_first_calls_of_a_process_may_be_captured_in_every_batch(batch):
    text = edges.CAPTURE.replace("torch.randn(4, 3, 40, 40", "torch.randn(%d, 3, 40, 40" % batch).replace("4, 3, 40, 40)", "%d, 3, 40, 40)" % batch)
    text = text.replace("scratch_bytes(4, 3,", "scratch_bytes(%d, 3," % batch)
    assert text.count("%d, 3, 40, 40" % batch) >= 4
    # a table of which the kernels need more shared memory than they have without asking
    text = text.replace("700", "9000")
    r = subprocess.run([sys.executable, "-c", text % edges.ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


def test_bias_windows_of_a_large_batch():
    """Windows of 49 positions, 4096 of them with 4 heads, 169 buckets: the map of a windowed backbone."""
    side, n = 7, 169
    at = torch.arange(side)
    y, x = torch.meshgrid(at, at, indexing="ij")
    y, x = y.reshape(-1), x.reshape(-1)
    buckets = ((y[:, None] - y[None] + side - 1) * (2 * side - 1) + x[:, None] - x[None] + side - 1).to(torch.int32).cuda()
    for batch, heads in ((4096, 4), (256, 16), (64, 32)):
        scores = base._normal((batch, heads, 49, 49), torch.bfloat16, "s", batch)
        table = base._normal((n, heads), torch.float32, "t", heads)
        out = torch.empty_like(scores)
        s2a.s2a_relbias_fwd(scores, table, buckets, out, batch, heads, 49, 49)
        base._done()
        want = scores.double() + table.double()[buckets.long()].permute(2, 0, 1)
        base._inside(out, want, (U + base.HALF[torch.bfloat16] * (1 + U)) * want.abs(), "bias")
        g = torch.randint(-1, 2, scores.shape, generator=base._gen("g", batch), device="cuda").bfloat16()
        exact = torch.zeros((n, heads), dtype=torch.float64, device="cuda")
        exact.index_add_(0, buckets.long().reshape(-1), g.double().sum(0).reshape(heads, -1).t().contiguous())
        # whole numbers, of which a bucket has at most 4096 * 49 in size: every sum is exact
        assert torch.equal(_grad(g, buckets, n).double(), exact)
