"""Host-side checks of layer norm, dropout and the relative position bias that need no GPU: size helpers, refusals
(all of them before any launch, so they are safe without a device), the dropout threshold, and the bucket of a distance
against whole-number arithmetic."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2503_08154_b200 import binding, build

F32, BF16 = 0, 1
OK, NULL, SHAPE, ALIGN, DTYPE, OVERLAP, VALUE = 0, 1, 2, 3, 4, 8, 9
A, B, C, D, E = 0x100000, 0x200000, 0x300000, 0x400000, 0x500000   # far apart, never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_value_status_string(lib):
    assert "VALUE" in binding.status_string(VALUE)


def _norm_fwd(lib, x=A, gamma=B, beta=B, y=C, stats=D, rows=0, L=64, xs=64, ys=64, eps=1e-6, dt=F32, wdt=F32):
    return lib.s2a_layernorm_fwd(x, gamma, beta, y, stats, rows, L, xs, ys, eps, dt, wdt, None)


def test_norm_forward_refusals(lib):
    assert _norm_fwd(lib) == OK                                    # no rows: nothing to do
    assert _norm_fwd(lib, dt=2) == DTYPE and _norm_fwd(lib, wdt=-1) == DTYPE
    assert _norm_fwd(lib, L=0) == SHAPE and _norm_fwd(lib, L=1 << 31) == SHAPE
    assert _norm_fwd(lib, rows=2, ys=63) == SHAPE                  # output rows that would overlap each other
    assert _norm_fwd(lib, rows=1 << 40, xs=1 << 40) == SHAPE       # not addressable
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _norm_fwd(lib, eps=eps) == VALUE
    assert _norm_fwd(lib, rows=2, x=None) == NULL and _norm_fwd(lib, rows=2, y=None) == NULL
    assert _norm_fwd(lib, rows=2, x=A + 2) == ALIGN and _norm_fwd(lib, rows=2, y=C + 1) == ALIGN
    assert _norm_fwd(lib, rows=2, stats=D + 4) == ALIGN and _norm_fwd(lib, rows=2, gamma=B + 1) == ALIGN
    assert _norm_fwd(lib, rows=2, x=A + 1, dt=BF16) == ALIGN


def test_norm_overlap_rules(lib):
    # a partial overlap, the same start under another stride, and rows of one stride that reach into each other
    assert _norm_fwd(lib, rows=4, x=A, y=A + 128) == OVERLAP
    assert _norm_fwd(lib, rows=4, x=A + 128, y=A) == OVERLAP
    assert _norm_fwd(lib, rows=4, x=A, xs=128, y=A) == OVERLAP
    assert _norm_fwd(lib, rows=4, x=A, xs=128, ys=128, y=A + 4 * 63) == OVERLAP
    assert _norm_fwd(lib, rows=4, x=A + 4 * 128, xs=128, ys=128, y=A + 4) == OVERLAP
    g, s = A, D
    bwd = lambda gin, xp=B, gs=64, os=64: lib.s2a_layernorm_bwd(g, xp, None, s, gin, E, E, None, 4, 64, gs, 64, os, F32, F32, None)
    assert bwd(C) == NULL                                          # weight gradients need scratch
    assert lib.s2a_layernorm_bwd(g, B, None, s, A + 64, None, None, None, 4, 64, 64, 64, 64, F32, F32, None) == OVERLAP
    assert lib.s2a_layernorm_bwd(g, B, None, s, B + 64, None, None, None, 4, 64, 64, 64, 64, F32, F32, None) == OVERLAP


def test_norm_backward_refusals(lib):
    def bwd(g=A, x=B, gamma=C, stats=D, gin=E, gg=C, gb=C, scratch=0x600000, rows=3, L=64, gs=64, xs=64, os=64, dt=F32, wdt=F32):
        return lib.s2a_layernorm_bwd(g, x, gamma, stats, gin, gg, gb, scratch, rows, L, gs, xs, os, dt, wdt, None)

    assert bwd(dt=7) == DTYPE and bwd(wdt=7) == DTYPE and bwd(L=0) == SHAPE and bwd(os=60) == SHAPE
    for name in ("g", "x", "stats", "gin"):
        assert bwd(**{name: None}) == NULL
    assert bwd(stats=D + 4) == ALIGN and bwd(scratch=0x600008) == ALIGN and bwd(gg=C + 2) == ALIGN
    assert bwd(g=A + 1, dt=BF16) == ALIGN
    # no rows and frozen weights: nothing to write
    assert bwd(rows=0, gg=None, gb=None, scratch=None) == OK


def test_norm_scratch(lib):
    f = binding.layernorm_scratch_bytes
    assert f(5, 0) == 0 and f(5, 1 << 31) == 0
    for L in (1, 31, 768, 1025, 4096, 16384, 16385, 100000):
        last = 0
        for rows in (0, 1, 7, 8, 9, 100, 1000, 10 ** 6):
            n = f(rows, L)
            assert n % (8 * L) == 0 and last <= n <= 888 * L * 4 and n >= 8 * L
            last = n


def test_dropout_threshold(lib):
    t = binding.dropout_threshold
    assert t(0.0) == 0 and t(1.0) == 65536 and t(0.5) == 32768 and t(0.1) == 6554
    assert t(1e-9) == 0 and t(1 - 1e-9) == 65536
    for i in range(0, 2048):
        p = i / 2048
        assert t(p) == round(65536 * p)


def test_dropout_refusals(lib):
    def f(x=A, r=B, y=C, n=64, rng=D, p=0.1, dt=F32):
        return lib.s2a_dropout_fwd(x, r, y, n, rng, 3, p, dt, None)

    assert f(n=0) == OK and f(dt=3) == DTYPE
    for p in (-0.1, 1.1, float("nan")):
        assert f(p=p) == VALUE
    for name in ("x", "y", "rng"):
        assert f(**{name: None}) == NULL
    assert f(x=A + 4) == ALIGN and f(r=B + 4) == ALIGN and f(y=C + 8) == ALIGN and f(rng=D + 4) == ALIGN
    assert f(y=A + 128) == OVERLAP and f(y=B + 128) == OVERLAP
    assert f(n=1 << 61) == SHAPE
    assert lib.s2a_dropout_bwd(A, A + 64, 64, D, 3, 0.1, F32, None) == OVERLAP
    assert lib.s2a_dropout_bwd(A, None, 64, D, 3, 0.1, F32, None) == NULL


def test_bias_refusals(lib):
    def f(x=A, table=B, buckets=C, y=D, batch=2, heads=3, tq=5, tk=7, n=8, dt=F32, wdt=F32, by=0):
        return lib.s2a_relbias_fwd(x, table, buckets, by, y, batch, heads, tq, tk, n, dt, wdt, None)

    assert f(batch=0) == OK and f(tq=0) == OK and f(tk=0, by=1) == OK
    assert f(dt=2) == DTYPE and f(wdt=2) == DTYPE
    assert f(heads=0) == SHAPE and f(heads=65536) == SHAPE and f(n=0) == SHAPE and f(n=32769) == SHAPE
    assert f(tq=1 << 21, tk=1 << 20) == SHAPE and f(batch=1 << 31) == SHAPE
    assert f(batch=1 << 30, heads=65535, tq=1 << 20, tk=1 << 20) == SHAPE
    for name in ("x", "table", "buckets", "y"):
        assert f(**{name: None}) == NULL
    assert f(x=A + 4) == ALIGN and f(y=D + 8) == ALIGN and f(table=B + 2) == ALIGN and f(buckets=C + 2) == ALIGN
    assert f(y=A + 16) == OVERLAP

    def g(go=A, buckets=B, table=C, scratch=D, batch=2, heads=3, tq=5, tk=7, n=8, dt=F32, wdt=F32):
        return lib.s2a_relbias_bwd(go, buckets, 0, table, scratch, batch, heads, tq, tk, n, dt, wdt, None)

    assert g(dt=2) == DTYPE and g(heads=0) == SHAPE and g(n=1 << 20) == SHAPE
    for name in ("go", "buckets", "table", "scratch"):
        assert g(**{name: None}) == NULL
    assert g(go=A + 2) == ALIGN and g(scratch=D + 8) == ALIGN and g(buckets=B + 1) == ALIGN


def test_bias_scratch(lib):
    f = binding.relbias_scratch_bytes
    assert f(0, 12, 197, 197, 732) == 0 and f(2, 0, 5, 5, 8) == 0 and f(2, 3, 5, 5, 40000) == 0
    for batch, heads, tq, tk, n in ((64, 12, 197, 197, 732), (1, 1, 1, 1, 1), (2, 16, 2048, 2048, 32), (3, 65535, 1, 9, 64),
                                    (1, 2, 50, 50, 32768)):
        b = f(batch, heads, tq, tk, n)
        assert b % (4 * n) == 0 and 4 * n * heads <= b <= 4 * max(1 << 22, heads * n)


def _bucket(d, n_buckets, max_distance, bidirectional):
    """The definition in whole numbers: bucket e + j of a side starts at n >= e (m / e)^(j / w), i.e. n^w e^j >= e^w m^j."""
    side = n_buckets // 2 if bidirectional else n_buckets
    e = side // 2
    w = side - e
    n = abs(d) if bidirectional else max(-d, 0)
    if n < e:
        u = n
    else:
        j = 0
        while j + 1 < w and n ** w * e ** (j + 1) >= e ** w * max_distance ** (j + 1):
            j += 1
        u = e + j
    return u + (side if bidirectional and d > 0 else 0)


@pytest.mark.parametrize("n_buckets,max_distance,bidirectional",
                         [(32, 128, True), (32, 128, False), (8, 16, True), (4, 2, True), (2, 7, False), (64, 1000, True),
                          (33, 257, False), (32, 17, False), (16, 4096, False), (130, 333, True)])
def test_distance_buckets(lib, n_buckets, max_distance, bidirectional):
    first, count = -2 * max_distance - 9, 4 * max_distance + 19
    got = binding.log_buckets(first, count, n_buckets, max_distance, bidirectional)
    want = [_bucket(d, n_buckets, max_distance, bidirectional) for d in range(first, first + count)]
    assert got.dtype == torch.int32 and got.tolist() == want
    # a window of the distances is the same window of the buckets, wherever it begins
    for lo, m in ((-3, 7), (1, 5), (max_distance - 2, 4), (-max_distance, 1), (0, 1), (5, 0)):
        got = binding.log_buckets(lo, m, n_buckets, max_distance, bidirectional)
        assert got.tolist() == [_bucket(d, n_buckets, max_distance, bidirectional) for d in range(lo, lo + m)]


@pytest.mark.parametrize("n_buckets,max_distance,j,n",
                         [(512, 1073822369, 223, 150392436), (512, 1074060938, 222, 141722813), (32768, 2147483647, 16383, 2145937485)])
def test_distance_buckets_where_a_border_is_almost_a_whole_number(lib, n_buckets, max_distance, j, n):
    """Border j of the first two lies 5.8e-8 and 4.8e-8 above n, within 1e-15 of it: n is still in the bucket before.  The last is the
    largest table's last border, the nearest distances to it."""
    for k in range(-2, 3):
        got = binding.log_buckets(-(n + k), 1, n_buckets, max_distance, False)
        assert got.tolist() == [_bucket_at(n + k, n_buckets, max_distance, j)], k


def _bucket_at(n, n_buckets, max_distance, j):
    """`_bucket` for one side and an n known to lie by border j: which side of it n is on, in whole numbers."""
    e = n_buckets // 2
    w = n_buckets - e
    f = math.gcd(j, w)          # n >= e (m / e)^(j / w), with the fraction in lowest terms
    j, w = j // f, w // f
    return e + j * f - (0 if n ** w >= e ** (w - j) * max_distance ** j else 1)


@pytest.mark.parametrize("n_buckets,max_distance,bidirectional", [(128, 64 * 4 ** 12, False), (32, 8 * 3 ** 8, True), (96, 48 * 5 ** 6, False), (64, 18 * 32, False)])
def test_distance_buckets_where_borders_are_whole_numbers(lib, n_buckets, max_distance, bidirectional):
    side = n_buckets // 2 if bidirectional else n_buckets
    e = side // 2
    for j in range(1, side - e):
        near = round(e * (max_distance / e) ** (j / (side - e)))
        first = near - 3
        got = binding.log_buckets(-(first + 6), 7, n_buckets, max_distance, bidirectional).tolist()
        assert got == [_bucket(-n, n_buckets, max_distance, bidirectional) for n in range(first + 6, first - 1, -1)], j


def test_distance_bucket_refusals(lib):
    out = (ctypes.c_int32 * 4)()
    f = lambda *a: lib.s2a_relbias_log_buckets(out, *a)
    assert f(0, 4, 33, 128, 1) == SHAPE and f(0, 4, 2, 128, 1) == SHAPE and f(0, 4, 1, 128, 0) == SHAPE
    assert f(0, 4, 1 << 16, 1 << 20, 0) == SHAPE
    assert f(0, 4, 32, 8, 1) == VALUE and f(0, 4, 32, 0, 0) == VALUE and f(0, 4, 32, 1 << 31, 0) == VALUE
    assert f(1 << 41, 4, 32, 128, 0) == VALUE and f(-(1 << 41), 4, 32, 128, 0) == VALUE
    assert lib.s2a_relbias_log_buckets(None, 0, 4, 32, 128, 1) == NULL
    assert lib.s2a_relbias_log_buckets(None, 0, 0, 32, 128, 1) == OK


def test_binding_refuses_host_tensors(lib):
    x, w = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises(binding.S2AError, match="CUDA"):
        binding.s2a_layernorm_fwd(x, w, w, x, None, 8, 1e-6)
    with pytest.raises(binding.S2AError, match="CUDA"):
        binding.s2a_dropout_bwd(x, x, torch.zeros(2, dtype=torch.int64), 0, 0.5)
    with pytest.raises(binding.S2AError, match="CUDA"):
        binding.s2a_relbias_bwd(x, torch.zeros(1, dtype=torch.int32), w, w, 1, 1, 4, 8)


def test_row_strides():
    """What counts as evenly spaced rows (host logic, on CPU tensors)."""
    rows = binding._rows
    t = torch.zeros(6, 5, 8)
    assert rows(t, 30, 8, "t") == 8 and rows(t, 60, 4, "t") == 4
    assert rows(t[:, 0], 6, 8, "t") == 40 and rows(t[:, 1:2], 6, 8, "t") == 40 and rows(t[::2, 3], 3, 8, "t") == 80
    assert rows(t[0], 5, 8, "t") == 8 and rows(t[:1, :1], 1, 8, "t") == 8 and rows(t[:, :, :4], 30, 4, "t") == 8
    assert rows(t[:, ::1, 2:6], 30, 4, "t") == 8 and rows(torch.zeros(8).expand(3, 8), 3, 8, "t") == 0
    for bad, n, L in ((t[:, :2], 12, 8), (t.transpose(1, 2), 48, 5), (t[..., ::2], 30, 4), (t[:, 0], 12, 4), (t, 29, 8)):
        with pytest.raises(binding.S2AError):
            rows(bad, n, L, "t")


def test_no_new_kernel_uses_floating_atomics():
    here = os.path.join(os.path.dirname(binding.__file__), "csrc")
    for name in ("s2a_layernorm.cu", "s2a_dropout.cu", "s2a_relbias.cu"):
        assert not re.search(r"\batomic(Add|CAS|Exch)\b|red\.", open(os.path.join(here, name)).read()), name
