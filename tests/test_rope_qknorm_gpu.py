"""GPU parity of rotary positions and of the norms of queries and keys against plain 64-bit forms.

Tolerances, with u = 2^-24 (half a step of binary32) and h the half step of the output type (2^-8 for bfloat16, u for binary32):

* rotation: the phase loses less than 2^-32 of a turn (1.5e-9 rad), its conversion u pi / 4, the sine and cosine one step
  of binary32 (2 u) and their product with the scale u: below 4 u |scale| each.  Two products and a sum add 2 u each:
  d = 6 u |scale| (|a| + |b|), and h |out| for the output.
* norm: a sum of squares goes through at most 16 + 5 additions (16 elements a lane, five steps of shuffles), and a product each:
  22 u relative; rstd has half of it, and 3 u for the mean's product, eps and the reciprocal root: 14 u.  x rstd gamma: 16 u.
* backward: u' = the gradient turned back (d), a = u' gamma: d |gamma| + u |a|; the mean of a xhat: (sum |da| |x| + 23 u
  sum |a x|) rstd / D + 15 u of itself; grad = (a - xhat mean) rstd with 14 u of it for rstd and 18 u of xhat mean.
* grad_gamma: terms u' xhat are off by d |xhat| + 17 u |u' xhat|; a term passes through at most as many additions as a
  lane has rows, fewer than the rows over 32 / lanes at these sizes, then 256 in a CTA, 19 of the CTAs and 16 warps.
Results below the normal range may be flushed: + 2^-126.
"""
import math
import random

import pytest
import torch

from paper_2503_08154_b200 import binding as s2a

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -126
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TAU = 2 * math.pi


def _gen(*key):
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * ord(c) for i, c in enumerate(repr(key))))


def _normal(shape, dtype, *key, scale=1.0):
    return (torch.randn(shape, generator=_gen(*key), device="cuda") * scale).to(dtype)


def _inside(got, want, tol, what):
    got, want, tol = got.double(), want.double(), (tol.double() + TINY).expand(want.shape)
    bad = ~((got - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError("%s: %d of %d outside tolerance, first at %s: got %r want %r tol %r"
                             % (what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(tol[i])))


def _done():
    torch.cuda.synchronize()
    assert s2a.s2a_device_error() == 0


class Placed:
    """[batch, tokens, heads, dim] in a buffer of its own: `order` of the dimensions, gaps behind rows and heads, an offset;
    what is not part of the tensor is checked to stay."""

    def __init__(self, shape, dtype, rng, key, order=None, plain=False):
        b, t, h, d = shape
        sizes = {"b": b, "t": t, "h": h}
        order = order or rng.choice(["bth", "bht", "tbh", "hbt"])
        gap = 0 if plain else rng.choice([0, 0, 1, 8, 16])
        step, strides = d + gap, {}
        for name in reversed(order):
            strides[name] = step
            step = step * sizes[name] + (0 if plain else rng.choice([0, 0, 8, 3]))
        offset = 0 if plain else rng.choice([0, 0, 8, 1, 2])
        self.buf = _normal((step + offset + 8,), dtype, "buf", key)
        self.view = torch.as_strided(self.buf, shape, (strides["b"], strides["t"], strides["h"], 1), offset)
        mark = torch.ones_like(self.buf, dtype=torch.bool)
        torch.as_strided(mark, shape, (strides["b"], strides["t"], strides["h"], 1), offset).fill_(False)
        self.rest, self.before = mark, self.buf[mark].clone()

    def untouched(self):
        assert torch.equal(self.buf[self.rest], self.before), "elements outside the tensor were written"


def _angles(table, positions, batch, tokens, first=0):
    """[batch, tokens, 1, pairs] in 64 bits, from the table's whole numbers: exact."""
    turns = [(a % (1 << 64), b) for a, b in table.cpu().tolist()]
    if positions is None:
        pos = torch.arange(first, first + tokens).expand(1, batch, tokens)
    else:
        p = positions.cpu().long()
        pos = p.expand(1, batch, tokens) if p.dim() < 3 else p
    distinct, back = torch.unique(pos, return_inverse=True)
    out = torch.empty((batch, tokens, 1, len(turns)), dtype=torch.float64)
    values = distinct.tolist()
    for i, (turn, axis) in enumerate(turns):
        axis = min(axis, pos.shape[0] - 1) if axis >= 0 else pos.shape[0] - 1
        part = torch.tensor([((v * turn) % (1 << 64)) / 2.0 ** 64 for v in values], dtype=torch.float64)
        out[:, :, 0, i] = part[back[axis]]
    return out.cuda() * TAU


def _turn(x, angle, scale, interleaved, back=False):
    """The rotated x and the magnitude |a| + |b| of each output (zero where nothing turns), in 64 bits."""
    x = x.double()
    rot = 2 * angle.shape[-1]
    c, s = torch.cos(angle) * scale, torch.sin(angle) * scale * (-1 if back else 1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v, m = a * c - b * s, a * s + b * c, abs(scale) * (a.abs() + b.abs())

    def join(p, q, tail):
        front = torch.stack([p, q], -1).flatten(-2) if interleaved else torch.cat([p, q], -1)
        return torch.cat([front, tail], -1)

    return join(u, v, x[..., rot:]), join(m, m, torch.zeros_like(x[..., rot:]))


def _norm_fwd(x, gamma, eps, angle, scale, interleaved):
    x = x.double()
    gamma = torch.ones(x.shape[-1], dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    rstd = ((x * x).mean(-1, keepdim=True) + eps) ** -0.5
    y, m = _turn(x * rstd * gamma, angle, scale, interleaved)
    return y, 22 * U * m + 16 * U * y.abs()


def _norm_bwd(g, x, gamma, eps, angle, scale, interleaved):
    g, x = g.double(), x.double()
    D = x.shape[-1]
    gamma = torch.ones(D, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    rstd = ((x * x).mean(-1, keepdim=True) + eps) ** -0.5
    u, m = _turn(g, angle, scale, interleaved, back=True)
    d = 6 * U * m
    a, xhat = u * gamma, x * rstd
    da = d * gamma.abs() + U * a.abs()
    mean = (a * xhat).mean(-1, keepdim=True)
    dmean = ((da * x.abs()).sum(-1, keepdim=True) + 23 * U * (a * x).abs().sum(-1, keepdim=True)) * rstd / D + 15 * U * mean.abs()
    grad = (a - xhat * mean) * rstd
    tol = rstd * (da + xhat.abs() * dmean + 18 * U * (xhat * mean).abs()) + 14 * U * grad.abs()
    terms = u * xhat
    rows = x.numel() // D
    lanes = -(-D // 16)
    depth = -(-rows // (32 // lanes)) + 256 + 28 + 32
    dg = (d * xhat.abs() + (17 + depth) * U * terms.abs()).sum((0, 1, 2))
    return grad, tol, terms.sum((0, 1, 2)), dg


def _run_case(seed, norm):
    rng = random.Random(seed)
    dt, wt = rng.choice(list(DT.values())), rng.choice(list(DT.values()))
    batch, tokens = rng.choice([(1, 1), (5, 1), (1, 33), (2, 17), (3, 100), (64, 1), (2, 700)])
    heads = rng.choice([(1, 0), (1, 1), (4, 4), (8, 2), (5, 3), (12, 12), (32, 8), (3, 1)])
    D = rng.choice([1, 2, 7, 8, 16, 24, 40, 64, 64, 72, 80, 96, 100, 128, 128, 129, 160, 192, 256, 320, 512])
    choices = [r for r in (D // 2 * 2, D // 4 * 2, D // 8 * 4, D // 16 * 8, 2) if 2 <= r <= D] or [0]
    rot = rng.choice(choices + ([0] if norm else []))
    if rot == 0 and not norm:
        D, rot = 2, 2
    inter = rng.random() < 0.5
    axes = rng.choice([a for a in (1, 1, 2, 3) if rot and rot // 2 % a == 0] or [1])
    scale = rng.choice([1.0, 1.0, 1.2772])
    if rot:
        table = s2a.rope_table(rot, scaling=rng.choice(["none", "linear", "base", "parts"]), factor=8.0, original_length=4096, axes=axes).cuda()
    else:
        table = None
    span = rng.choice([3, 1000, 2 ** 31 - 1])
    form = rng.choice([1, 2, 3]) if axes == 1 else 3
    shape = {1: (tokens,), 2: (batch, tokens), 3: (axes, batch, tokens)}[form]
    positions = torch.randint(-span if rng.random() < 0.3 else 0, span, shape, generator=_gen("pos", seed), device="cuda", dtype=torch.int32)
    first = 0
    if axes == 1 and rng.random() < 0.2:
        positions, first = None, rng.choice([0, 77, 2 ** 33])
    plain = rng.random() < 0.4
    order = rng.choice(["bth", "bht", None])
    make = lambda n, key: Placed((batch, tokens, n, D), dt, rng, (key, seed), order, plain)  # noqa: E731
    angle = (_angles(table, positions, batch, tokens, first) if rot else torch.zeros((batch, tokens, 1, 0), dtype=torch.float64, device="cuda"))
    q, k, oq, ok, gq, gk = (make(max(n, 1), key) for n, key in zip([*heads] * 3, "abcdef"))
    if heads[1] == 0:
        k = ok = gk = None
    v = lambda p: None if p is None else p.view  # noqa: E731
    rest = (positions, table)
    both = [(x, o, g) for x, o, g in ((q, oq, gq), (k, ok, gk)) if x is not None]
    if not norm:
        for call, back in ((s2a.s2a_rope_fwd, False), (s2a.s2a_rope_bwd, True)):
            call(v(q), v(k), v(oq), v(ok), *rest, scale=scale, interleaved=inter, first=first)
            _done()
            for x, o, _ in both:
                want, m = _turn(x.view, angle, scale, inter, back)
                d = 6 * U * m
                _inside(o.view, want, d + HALF[dt] * (want.abs() + d), "rotation")
                assert torch.equal(o.view[..., rot:], x.view[..., rot:])
                o.untouched()
        return
    eps = rng.choice([1e-6, 1e-5, 0.1])
    gamma = [_normal((D + 3,), wt, "gamma", i, seed)[rng.choice([0, 1, 3]):][:D] if rng.random() < 0.8 else None for i in range(2)]
    s2a.s2a_qknorm_rope_fwd(v(q), v(k), *gamma, v(oq), v(ok), *rest, eps, scale=scale, interleaved=inter, first=first)
    _done()
    for i, (x, o, _) in enumerate(both):
        want, tol = _norm_fwd(x.view, gamma[i], eps, angle, scale, inter)
        _inside(o.view, want, tol + HALF[dt] * (want.abs() + tol), "norm")
        o.untouched()
    grads = [torch.full((D + 1,), 7.0, dtype=wt, device="cuda")[1:] if rng.random() < 0.8 else None for _ in range(2)]
    need = s2a.qknorm_rope_scratch_bytes(batch, tokens, heads[0], heads[1], D)
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xFF) if any(t is not None for t in grads) else None
    s2a.s2a_qknorm_rope_bwd(v(gq), v(gk), v(q), v(k), *gamma, v(oq), v(ok), *grads, scratch, *rest, eps, scale=scale, interleaved=inter,
                            first=first)
    _done()
    for i, (x, o, g) in enumerate(both):
        want, tol, sums, dsums = _norm_bwd(g.view, x.view, gamma[i], eps, angle, scale, inter)
        _inside(o.view, want, tol + HALF[dt] * (want.abs() + tol), "gradient")
        o.untouched()
        if grads[i] is not None:
            _inside(grads[i], sums, dsums + HALF[wt] * (sums.abs() + dsums), "weights' gradient")
    if heads[1] == 0 and grads[1] is not None:
        assert not grads[1].any()      # a sum over no rows


@pytest.mark.parametrize("seed", range(70))
def test_rotation_walk(seed):
    _run_case(seed, norm=False)


@pytest.mark.parametrize("seed", range(100, 190))
def test_norm_walk(seed):
    _run_case(seed, norm=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,heads,D", [(1, (32, 8), 128), (197, (12, 12), 64), (1, (1, 1), 2), (4099, (2, 1), 128)])
def test_packed_buffer_and_in_place(tokens, heads, D, dtype):
    """Queries, keys and values side by side in one buffer: the values stay, in place gives what another output gives."""
    dt, batch = DT[dtype], 3
    width = heads[0] + 2 * heads[1]
    buf = _normal((batch, tokens, width, D), dt, "packed", tokens, D)
    q, k = buf[:, :, :heads[0]], buf[:, :, heads[0]:heads[0] + heads[1]]
    table = s2a.rope_table(D).cuda()
    pos = torch.arange(5, 5 + tokens, dtype=torch.int32, device="cuda")
    gamma = _normal((D,), torch.float32, "g", D)
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    s2a.s2a_qknorm_rope_fwd(q, k, gamma, gamma, oq, ok, pos, table, 1e-6)
    rq, rk = torch.empty_like(q), torch.empty_like(k)
    s2a.s2a_rope_fwd(q, k, rq, rk, pos, table)
    again = buf.clone()
    a, b = again[:, :, :heads[0]], again[:, :, heads[0]:heads[0] + heads[1]]
    s2a.s2a_qknorm_rope_fwd(a, b, gamma, gamma, a, b, pos, table, 1e-6)
    _done()
    assert torch.equal(a, oq) and torch.equal(b, ok) and torch.equal(again[:, :, sum(heads):], buf[:, :, sum(heads):])
    again = buf.clone()
    a, b = again[:, :, :heads[0]], again[:, :, heads[0]:heads[0] + heads[1]]
    s2a.s2a_rope_fwd(a, b, a, b, None, table, first=5)
    _done()
    assert torch.equal(a, rq) and torch.equal(b, rk) and torch.equal(again[:, :, sum(heads):], buf[:, :, sum(heads):])
    # backward into the gradient's place, and into x's
    g = _normal(buf.shape, dt, "grad", tokens, D)
    gq, gk = g[:, :, :heads[0]], g[:, :, heads[0]:heads[0] + heads[1]]
    scratch = torch.empty(s2a.qknorm_rope_scratch_bytes(batch, tokens, *heads, D), dtype=torch.uint8, device="cuda")
    results = []
    for place in ("apart", "gradient", "x"):
        x2, g2 = buf.clone(), g.clone()
        part = lambda t: (t[:, :, :heads[0]], t[:, :, heads[0]:heads[0] + heads[1]])  # noqa: E731
        out = {"apart": (oq, ok), "gradient": part(g2), "x": part(x2)}[place]
        sums = [torch.empty(D, device="cuda") for _ in range(2)]
        s2a.s2a_qknorm_rope_bwd(*part(g2), *part(x2), gamma, gamma, *out, *sums, scratch, pos, table, 1e-6)
        _done()
        results.append([t.clone() for t in (*out, *sums)])
    for other in results[1:]:
        assert all(torch.equal(p, r) for p, r in zip(results[0], other))
    assert gq.shape == oq.shape and gk.shape == ok.shape


def test_turning_back_and_lengths():
    """Backward undoes forward, and a pair keeps its length, at positions up to the ends of the type."""
    x = _normal((2, 6, 3, 64), torch.float32, "x")
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32, device="cuda")
    table = s2a.rope_table(64).cuda()
    for inter in (False, True):
        y, z = torch.empty_like(x), torch.empty_like(x)
        s2a.s2a_rope_fwd(x, None, y, None, pos, table, interleaved=inter)
        s2a.s2a_rope_bwd(y, None, z, None, pos, table, interleaved=inter)
        _done()
        assert torch.equal(y[:, 0], x[:, 0])
        assert float((z - x).abs().max()) <= 2 * 6 * U * 2 * float(x.abs().max()) * 1.5
        # the same turns one position apart: scores depend on the distance alone
        assert torch.allclose(y.square().sum(-1), x.square().sum(-1), rtol=1e-5)


def test_positions_come_before_first():
    """With positions, `first` is not looked at; without rotation nothing of them is."""
    x = _normal((2, 9, 3, 32), torch.float32, "x")
    pos = torch.randint(0, 500, (2, 9), generator=_gen("p"), device="cuda", dtype=torch.int32)
    table = s2a.rope_table(32).cuda()
    y, z = torch.empty_like(x), torch.empty_like(x)
    s2a.s2a_rope_fwd(x, None, y, None, pos, table)
    s2a.s2a_rope_fwd(x, None, z, None, pos, table, first=77)
    _done()
    assert torch.equal(y, z)
    s2a.s2a_qknorm_rope_fwd(x, None, None, None, y, None, None, None, 1e-6)
    s2a.s2a_qknorm_rope_fwd(x, None, None, None, z, None, pos[:, :3], None, 1e-6, first=5)
    _done()
    assert torch.equal(y, z)


def test_a_table_of_the_callers_own_and_an_axis_beyond_the_last():
    x = _normal((1, 9, 2, 16), torch.float32, "x")
    pos = torch.randint(0, 50, (2, 1, 9), generator=_gen("p"), device="cuda", dtype=torch.int32)
    table = s2a.rope_table(16)
    table[:, 1] = torch.tensor([0, 1, 0, 1, 7, -1, 1 << 40, 0])
    y, z = torch.empty_like(x), torch.empty_like(x)
    s2a.s2a_rope_fwd(x, None, y, None, pos, table.cuda())
    table[:, 1] = torch.tensor([0, 1, 0, 1, 1, 1, 1, 0])
    s2a.s2a_rope_fwd(x, None, z, None, pos, table.cuda())
    _done()
    assert torch.equal(y, z)
    want, m = _turn(x, _angles(table, pos, 1, 9), 1.0, False)
    _inside(z, want, 6 * U * m + U * want.abs(), "own table")


@pytest.mark.parametrize("D", [16, 72, 128])
def test_rows_do_not_leak_into_their_neighbours(D):
    """NaN, infinities and the largest values stay in their rows; empty rows give zeros."""
    x = _normal((2, 5, 7, D), torch.bfloat16, "x", D)
    g = _normal((2, 5, 7, D), torch.bfloat16, "g", D)
    bad = (torch.arange(70) % 3 == 1).view(2, 5, 7).cuda()
    table = s2a.rope_table(D // 2 // 8 * 8).cuda()
    gamma = _normal((D,), torch.float32, "gamma", D)

    def both(x, g):
        y, d = torch.empty_like(x), torch.empty_like(x)
        s2a.s2a_qknorm_rope_fwd(x, None, gamma, None, y, None, None, table, 1e-6)
        s2a.s2a_qknorm_rope_bwd(g, None, x, None, gamma, None, d, None, None, None, None, None, table, 1e-6)
        _done()
        return y, d

    want = both(x, g)
    for poison in (float("nan"), float("inf"), 3e38, 0.0):
        xp, gp = x.clone(), g.clone()
        xp[bad] = poison
        got = both(xp, gp)
        for a, b in zip(got, want):
            assert torch.equal(a[~bad], b[~bad])
        if poison == 0.0:
            assert not got[0][bad].any() and bool(torch.isfinite(got[1]).all())
        if poison == 3e38:
            assert not got[0][bad].any()       # a sum of squares beyond binary32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,rot", [(40, 16), (128, 64), (11, 4), (24, 2)])
def test_what_does_not_turn_is_copied_bit_for_bit(D, rot, dtype):
    """Infinities, NaN and negative zeros behind the turning part stay what and where they are; so do those of a pair in their pair."""
    dt = DT[dtype]
    x = _normal((2, 3, 5, D), dt, "x", D)
    x[..., rot::2] = float("inf")
    x[..., rot + 1::3] = -0.0
    x[..., D - 1] = float("nan")
    x[0, :, :, 0] = float("inf")
    table = s2a.rope_table(rot).cuda()
    for inter in (False, True):
        y = torch.empty_like(x)
        s2a.s2a_rope_fwd(x, None, y, None, None, table, interleaved=inter)
        _done()
        kind = {2: torch.int16, 4: torch.int32}[dt.itemsize]
        assert torch.equal(y[..., rot:].contiguous().view(kind), x[..., rot:].contiguous().view(kind))
        pair = [0, 1] if inter else [0, rot // 2]
        others = [i for i in range(rot) if i not in pair]
        assert bool(torch.isfinite(y[..., others]).all()) and bool(torch.isfinite(y[1, ..., :rot]).all())
        assert not bool(torch.isfinite(y[0, ..., pair[0]]).any())


def test_broadcast_keys_and_shared_positions():
    """One key row expanded over heads and batch is read as it is; each copy has its own gradient."""
    one = _normal((1, 6, 1, 32), torch.bfloat16, "k")
    q = _normal((4, 6, 8, 32), torch.bfloat16, "q")
    table = s2a.rope_table(32).cuda()
    gamma = _normal((32,), torch.bfloat16, "gamma")
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    k = one.expand(4, 6, 8, 32)
    outs = []
    for keys, p in ((k, pos), (k.contiguous(), pos.expand(4, 6).contiguous()), (k, pos.expand(1, 4, 6))):
        oq, ok = torch.empty_like(q), torch.empty((4, 6, 8, 32), dtype=torch.bfloat16, device="cuda")
        s2a.s2a_qknorm_rope_fwd(q, keys, gamma, gamma, oq, ok, p, table, 1e-6)
        dq, dk = torch.empty_like(q), torch.empty_like(ok)
        sums = [torch.empty(32, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        scratch = torch.empty(s2a.qknorm_rope_scratch_bytes(4, 6, 8, 8, 32), dtype=torch.uint8, device="cuda")
        s2a.s2a_qknorm_rope_bwd(q, q, q, keys, gamma, gamma, dq, dk, *sums, scratch, p, table, 1e-6)
        _done()
        outs.append([oq, ok, dq, dk, *sums])
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_against_differences(interleaved):
    """Along random directions: the derivative of sum(w * forward) in 64 bits by central differences, whose error is below 1e-7 of
    the terms (steps of 1e-4: h^2 / 6 of third derivatives of order ten), against what backward gives in binary32."""
    shape, D = (2, 11, 3, 24), 24
    x, w = _normal(shape, torch.float32, "x"), _normal(shape, torch.float32, "w")
    gamma = 1 + 0.3 * _normal((D,), torch.float32, "gamma")
    table = s2a.rope_table(16).cuda()
    angle = _angles(table, None, 2, 11, 3)
    grad, sums = torch.empty_like(x), torch.empty(D, device="cuda")
    scratch = torch.empty(s2a.qknorm_rope_scratch_bytes(2, 11, 3, 0, D), dtype=torch.uint8, device="cuda")
    s2a.s2a_qknorm_rope_bwd(w, None, x, None, gamma, None, grad, None, sums, None, scratch, None, table, 1e-6, scale=1.1,
                            interleaved=interleaved, first=3)
    _done()

    def loss(x, gamma):
        return float((w.double() * _norm_fwd(x, gamma, 1e-6, angle, 1.1, interleaved)[0]).sum())

    for i in range(4):
        dx, dg = _normal(shape, torch.float64, "dx", i), _normal((D,), torch.float64, "dg", i)
        h = 1e-4
        numeric = (loss(x.double() + h * dx, gamma) - loss(x.double() - h * dx, gamma)) / (2 * h)
        terms = grad.double() * dx
        assert abs(numeric - float(terms.sum())) <= 1e-5 * float(terms.abs().sum())
        numeric = (loss(x, gamma.double() + h * dg) - loss(x, gamma.double() - h * dg)) / (2 * h)
        terms = sums.double() * dg
        assert abs(numeric - float(terms.sum())) <= 1e-5 * float(terms.abs().sum())


def test_empty_calls():
    table = s2a.rope_table(32).cuda()
    for shape in ((0, 5, 4, 32), (3, 0, 4, 32), (3, 5, 0, 32)):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        s2a.s2a_rope_fwd(x, x, x, x, None, table)
        sums = [torch.full((32,), 5.0, device="cuda") for _ in range(2)]
        scratch = torch.empty(s2a.qknorm_rope_scratch_bytes(*shape[:3], shape[2], 32), dtype=torch.uint8, device="cuda")
        s2a.s2a_qknorm_rope_bwd(x, x, x, x, None, None, x, x, *sums, scratch, None, table, 1e-6)
        _done()
        assert not sums[0].any() and not sums[1].any()


def test_same_call_same_bits_other_stream_and_replay():
    """Repeated calls write the same bits; a captured call follows positions that change between replays; two graphs with a scratch
    each run side by side."""
    q = _normal((4, 300, 8, 128), torch.bfloat16, "q")
    k = _normal((4, 300, 2, 128), torch.bfloat16, "k")
    g, gk = _normal(q.shape, torch.bfloat16, "g"), _normal(k.shape, torch.bfloat16, "gk")
    gamma = _normal((128,), torch.float32, "gamma")
    table = s2a.rope_table(128).cuda()
    pos = torch.arange(300, dtype=torch.int32, device="cuda")

    def buffers():
        return [torch.empty_like(q), torch.empty_like(k), torch.empty(128, device="cuda"), torch.empty(128, device="cuda"),
                torch.empty(s2a.qknorm_rope_scratch_bytes(4, 300, 8, 2, 128), dtype=torch.uint8, device="cuda")]

    def call(b, p):
        s2a.s2a_qknorm_rope_bwd(g, gk, q, k, gamma, gamma, *b[:4], b[4], p, table, 1e-6)

    first = buffers()
    call(first, pos)
    _done()
    for _ in range(3):
        again = buffers()
        call(again, pos)
        _done()
        assert all(torch.equal(a, b) for a, b in zip(first[:4], again[:4]))
    moving = pos.clone()
    graphs, kept = [], []
    for _ in range(2):
        b = buffers()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(b, moving)
        graphs.append((graph, stream))
        kept.append(b)
    for shift in (0, 1000):
        moving.copy_(pos + shift)
        torch.cuda.synchronize()
        for graph, stream in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        want = buffers()
        torch.cuda.synchronize()
        call(want, pos + shift)
        _done()
        for b in kept:
            assert all(torch.equal(x, y) for x, y in zip(b[:4], want[:4]))


@pytest.mark.parametrize("D,tokens,heads", [(64, 2368, (8, 0)), (40, 2368, (10, 0)), (64, 8 * 2368, (1, 0)), (128, 1184, (4, 4)), (2, 1500, (16, 16))])
def test_weights_gradients_are_added_up_in_64_bits(D, tokens, heads):
    """Rows of ones whose gradients are the same in all rows: a lane has one row (or a few, whose sums the numbers below have room for), and what is
    added over lanes, warps and CTAs must be exact but for the last rounding.  Numbers of 20 bits: the sum of up to 16 of them is exact in binary32, a
    CTA's sum is rounded once (1 u), and so is the result (1 u)."""
    g = torch.randint(1 << 19, 1 << 20, (D,), generator=_gen("terms", D), device="cuda").float()
    x = [torch.ones((1, tokens, h, D), device="cuda") for h in heads]
    y = torch.empty_like(x[0])
    s2a.s2a_qknorm_rope_fwd(x[0], None, None, None, y, None, None, None, 0.0)
    _done()
    rstd = y[0, 0, 0, 0]
    assert bool((y == rstd).all())
    terms = [g.expand_as(t).contiguous() for t in x]
    out = [torch.empty_like(t) for t in x]
    sums = [torch.empty(D, device="cuda") for _ in heads]
    scratch = torch.empty(s2a.qknorm_rope_scratch_bytes(1, tokens, *heads, D), dtype=torch.uint8, device="cuda")
    keys = heads[1] > 0
    s2a.s2a_qknorm_rope_bwd(terms[0], terms[1] if keys else None, x[0], x[1] if keys else None, None, None, out[0], out[1] if keys else None, sums[0],
                            sums[1] if keys else None, scratch, None, None, 0.0)
    _done()
    for s, h in zip(sums, heads):
        if h:
            want = (g * rstd).double() * (tokens * h)      # each term is rounded to binary32 as it is added to the lane's first
            assert float(((s.double() - want).abs() / want).max()) <= 2.01 * U + (0 if float(rstd) == 1 else 16 * U)
