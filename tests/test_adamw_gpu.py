"""GPU parity of the AdamW step and of the gradients' norm against plain 64-bit forms.

Tolerances, u = 2^-24.  g' = g * scale (* factor): 2 u.  m + (1 - b1)(g' - m): u (|g' - m| + |m'|) and the weight's rounding, below 4 u
(|m| + |g'|).  v: 2 u of each term and 4 u for g'^2: 8 u v'.  sqrt: half of that and 2 u (one step of the approximate root): 6 u.
The bias corrections: the logarithm's rounding and its product with the step's number change 1 - b^t by at most 2 u of itself, its
evaluation by 2 u, the root and the quotient by 2 u: 6 u.  The quotient of the two: 4 u.  The update is off by at most
24 u of itself and by what m is off; p by 3 u |p| more.  8-bit states come in with one rounding of the scale's quotient, one of the
product (3 u; twice that for v).  Codes: x = 448 |m| / largest is off by 40 u of itself; a code is the one of the exact x unless x (and the random
bits) lie within that of the border between two codes, and then a neighbour's.
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
E4 = torch.float8_e4m3fn


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


def _philox(block, count, seed):
    """Philox4x32-10 at counters (block, count) on Python's whole numbers."""
    low = 0xFFFFFFFF
    c = [block & low, block >> 32, count & low, (count >> 32) & low]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & low, (p0 >> 32) ^ c[3] ^ k[1], p0 & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def _fields(n, block0, rng, site, weights):
    """The 16 random bits of each of a tensor's n elements."""
    seed, offset = (v % (1 << 64) for v in rng)
    out = []
    for b in range(-(-n // 8)):
        words = _philox(32 * block0 + b + ((1 << 63) if weights else 0), (offset + site) % (1 << 64), seed)
        for w in words:
            out += [w & 0xFFFF, w >> 16]
    return torch.tensor(out[:n], dtype=torch.int64, device="cuda")


def _grid(x):
    """The distance of e4m3 values around x (64 bits, x >= 0)."""
    _, e = torch.frexp(x)
    return torch.exp2((e - 1).clamp(min=-6).double() - 3)


def _check_codes(got, x, bits, floor, what):
    """got: the code's magnitude, x: the exact value in 0 .. 448; floor: nothing above zero becomes zero."""
    got, slack = got.double(), 40 * U * x + 2.0 ** -149
    unit = _grid(x)
    t = x / unit
    if bits is None:
        want, edge = torch.round(t), ((t - torch.floor(t)) - 0.5).abs()
    else:
        add = (bits.double() + 0.5) / 65536
        want = torch.floor(t + add)
        edge = ((t + add) - torch.round(t + add)).abs()
    want = (want * unit).clamp(max=448.0)
    if floor:
        want = torch.where(x > 0, want.clamp(min=2.0 ** -9), want)
    # random bits see 20 bits of x below the kept ones
    near = edge <= slack / unit + (0 if bits is None else 2.0 ** -19)
    off = got != want
    assert not bool((off & ~near).any()), what
    assert bool(((got - want).abs() <= 2 * unit)[off].all()), what
    assert float(off.double().mean()) <= 0.01 + 2 / max(1, off.numel()), what


def _step(t, hyper, bits, decay, rate, clip=None):
    """The step in 64 bits from a tensor's state before it: p, m, v and their tolerances."""
    lr, number, scale, b1, b2, eps = hyper
    g = t["g"].double() * scale * (1.0 if clip is None else clip)
    m, v, p = t["m"].double(), t["v"].double(), t["p"].double()
    came_m = came_v = 0.0
    if bits == 8:
        spread = lambda s, n: (s.double() / 448).repeat_interleave(256)[:n]  # noqa: E731
        m, r = m * spread(t["ms"], m.numel()), v * spread(t["vs"], v.numel())
        v = r * r
        came_m, came_v = 3 * U * m.abs(), 7 * U * v
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    dm, dv = 4 * U * (m.abs() + g.abs()) + came_m, 8 * U * v2 + came_v
    lr = lr * rate
    root = v2.sqrt()
    den = root / math.sqrt(1 - b2 ** number) + eps
    update = lr / (1 - b1 ** number) * m2 / den
    p2 = p - lr * decay * p - update
    dp = 24 * U * update.abs() + lr / (1 - b1 ** number) * dm / den + 3 * U * p.abs() + U * p2.abs()
    return p2, m2, v2, dp, dm, dv


def _tensors(sizes, pdt, gdt, bits, rng, key, copies, spread=1.0):
    """One dict a tensor, each in a buffer of its own with guarded ends."""
    out = []
    for i, n in enumerate(sizes):
        off = rng.choice([0, 0, 0, 1, 3, 8])
        far = rng.choice([off, off, rng.choice([0, 2, 5])])
        grow = 10.0 ** (spread * rng.uniform(-3, 1))

        def place(values, at=off):
            buf = torch.full((n + at + 9,), 77.0, dtype=torch.float32, device="cuda").to(values.dtype)
            buf[at:at + n] = values
            return buf[at:at + n]

        t = {"p": place(_normal((n,), pdt, key, "p", i)), "g": place(_normal((n,), gdt, key, "g", i, scale=grow), far)}
        m = _normal((n,), torch.float32, key, "m", i, scale=0.3 * grow)
        r = _normal((n,), torch.float32, key, "r", i, scale=grow).abs() + 0.1 * grow
        if bits == 32:
            t |= {"m": place(m), "v": place(r * r)}
        else:
            for name, x in (("m", m), ("v", r)):
                rows = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
                top = rows.abs().amax(1)
                codes = (rows * (448 / top)[:, None]).to(E4).view(-1)[:n]
                t[name] = place(codes.view(torch.uint8)).view(E4)
                t[name + "s"] = top.clone()
        if copies:
            t["copy"] = place(torch.zeros(n, dtype=torch.bfloat16, device="cuda"))
        out.append(t)
    return out


def _plan(ts, bits, copies, decay=0.0, rate=1.0):
    col = lambda n: [t[n] for t in ts]  # noqa: E731
    scales = (col("ms"), col("vs")) if bits == 8 else (None, None)
    return s2a.adamw_plan(col("p"), col("g"), col("m"), col("v"), *scales, col("copy") if copies else None, weight_decay=decay,
                          lr_scale=rate)


def _clone(ts):
    return [{n: v.clone() for n, v in t.items()} for t in ts]


def _check_step(before, after, hyper, bits, decay, rate, rng=None, site=0, clip=None, pdt=torch.float32, block0=0):
    for i, (b, a) in enumerate(zip(before, after)):
        n = b["p"].numel()
        if n == 0:
            continue
        p, m, v, dp, dm, dv = _step(b, hyper, bits, decay[i], rate[i], clip)
        if pdt is torch.bfloat16 and rng is not None:
            _, e = torch.frexp(p.abs())
            unit = torch.exp2((e - 8).clamp(min=-133).double())
            t = p.abs() / unit + _fields(n, block0, rng, site, True).double() / 65536
            want = torch.floor(t) * unit * torch.sign(p)
            near = (t - torch.round(t)).abs() <= (dp + U * p.abs()) / unit + 2.0 ** -16
            off = a["p"].double() != want
            assert not bool((off & ~near).any()), "parameter rounded at random"
            assert bool(((a["p"].double() - want).abs() <= 2 * unit)[off].all())
        else:
            _inside(a["p"], p, dp + HALF[pdt] * (p.abs() + dp), "parameter %d" % i)
        if "copy" in b:
            _inside(a["copy"], p, dp + HALF[torch.bfloat16] * (p.abs() + dp), "copy")
        if bits == 32:
            _inside(a["m"], m, dm, "exp_avg %d" % i)
            _inside(a["v"], v, dv, "exp_avg_sq %d" % i)
        else:
            draws = None if rng is None else _fields(n, block0, rng, site, False)
            for name, x, d, bits_ in (("m", m, dm, draws), ("v", v.sqrt(), 6 * U * v.sqrt(),
                                                               None if draws is None else (draws % 256) * 256 + draws // 256)):
                top = torch.nn.functional.pad(x.abs(), (0, -n % 256)).view(-1, 256).amax(1)
                _inside(a[name + "s"], top, torch.nn.functional.pad(d, (0, -n % 256)).view(-1, 256).amax(1) + 8 * U * top, name + " scale")
                # the codes stand for x over the scale as it was written
                unit = (448 / a[name + "s"].double()).repeat_interleave(256)[:n]
                code = a[name].to(torch.float64)
                exact = (x.abs() * unit).clamp(max=448.0)
                slack = d * unit
                same = code.abs() > 0
                assert bool((torch.sign(code) == torch.sign(x))[same & (x.abs() > d)].all())
                extra = slack <= 40 * U * exact       # m near zero, where its own rounding is larger than its code's
                _check_codes(code.abs()[extra], exact[extra], None if bits_ is None else bits_[extra], name == "v", name + " codes")
        block0 += -(-n // 256)


CASES = [(p, g, bits, r) for p in ("f32", "bf16") for g in ("f32", "bf16") for bits in (32, 8) for r in (False, True)]


@pytest.mark.parametrize("pdt,gdt,bits,random_bits", CASES)
def test_step_over_many_tensors(pdt, gdt, bits, random_bits):
    """Sizes at which a lane, a block of 256 and a warp's chunk begin and end; odd offsets, parts at different ones."""
    rng = random.Random("%s%s%d%d" % (pdt, gdt, bits, random_bits))
    sizes = [1, 2, 7, 8, 9, 255, 256, 257, 0, 1023, 1024, 1025, 1031, 2048, 5000, 3, 12345, 8, 1]
    copies = pdt == "f32"
    ts = _tensors(sizes, DT[pdt], DT[gdt], bits, rng, (pdt, gdt, bits), copies)
    decay = [rng.choice([0.0, 0.1]) for _ in sizes]
    rate = [rng.choice([1.0, 0.5, 0.0]) for _ in sizes]
    before = _clone(ts)
    hyper = (1e-2, 7.0, 0.25, 0.9, 0.999, 1e-8)
    control = torch.tensor(hyper[:3], device="cuda")
    draws = (0x1234567890ABCDEF, (1 << 62) + 5)
    state = torch.tensor(draws, dtype=torch.int64, device="cuda") if random_bits else None
    ends = [{n: v._base.clone() if v._base is not None and v.dtype is not E4 else None for n, v in t.items()} for t in ts]
    s2a.s2a_adamw_step(_plan(ts, bits, copies, decay, rate), control, *hyper[3:], rng=state, site=3)
    _done()
    _check_step(before, ts, tuple(float(c) for c in control.tolist()) + hyper[3:], bits, decay, rate, draws if random_bits else None, 3, pdt=DT[pdt])
    for t, e in zip(ts, ends):      # nothing beside the tensors is written
        for n, whole in e.items():
            if whole is not None and t[n].numel():
                at = t[n].storage_offset()
                now = t[n]._base
                assert torch.equal(now[:at], whole[:at]) and torch.equal(now[at + t[n].numel():], whole[at + t[n].numel():])


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_in_a_row_with_the_clip_factor(bits):
    """Norm, factor and step three times over, by number: each against the formula from the state before it."""
    rng = random.Random(bits)
    sizes = [4096, 100, 70001, 256]
    ts = _tensors(sizes, torch.float32, torch.bfloat16, bits, rng, ("row", bits), False)
    plan = _plan(ts, bits, False, 0.01)
    control = torch.tensor([3e-3, 0.0, 2.0], device="cuda")
    clip = torch.empty(2, device="cuda")
    scratch = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda").fill_(0xFF)
    for number in range(1, 4):
        control[1] += 1
        before = _clone(ts)
        s2a.s2a_grad_norm(plan, control, 1.5, clip, scratch)
        s2a.s2a_adamw_step(plan, control, 0.8, 0.95, 1e-6, clip=clip)
        _done()
        norm = 2.0 * math.sqrt(sum(float(t["g"].double().square().sum()) for t in ts))
        assert abs(float(clip[0]) - norm) <= 1e-5 * norm and abs(float(clip[1]) - min(1.0, 1.5 / (norm + 1e-6))) <= 1e-5
        hyper = (float(control[0]), float(number), 2.0, 0.8, 0.95, 1e-6)
        _check_step(before, ts, hyper, bits, [0.01] * 4, [1.0] * 4, clip=float(clip[1]))


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_gradients_norm(gdt):
    """Sums of squares of eight are held in 32 bits (10 u relative), their sums in 64; over magnitudes whose squares are beyond binary32."""
    for scale in (1.0, 1e-25, 1e25, 3e37, 1e-38):
        for sizes in ([1], [5, 1031, 8, 0, 257], [300_007, 12, 4096], [0]):
            gs = [_normal((n + 3,), torch.float32, "g", n, scale=scale).to(DT[gdt])[i % 4:][:n] for i, n in enumerate(sizes)]
            plan = s2a.adamw_plan(None, gs, None, None)
            clip = torch.full((2,), 9.0, device="cuda")
            control = torch.tensor([0.0, 0.0, 0.125], device="cuda")
            scratch = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda").fill_(0xFF)
            s2a.s2a_grad_norm(plan, control, 2.0, clip, scratch)
            _done()
            norm = 0.125 * math.sqrt(sum(float(g.double().square().sum()) for g in gs))
            # 300,007 gradients of 3e37 have a norm of 300007^0.5 * 3e37 / 8 = 2e39: binary32 ends at 3.4e38, and it is an infinity
            if norm > torch.finfo(torch.float32).max:
                assert float(clip[0]) == math.inf
            else:
                assert abs(float(clip[0]) - norm) <= 8 * U * norm + TINY
            factor = min(1.0, 2.0 / (norm + 1e-6))
            assert abs(float(clip[1]) - factor) <= 8 * U * factor + TINY


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
@pytest.mark.parametrize("blocks", [2047, 2048, 2049, 11839, 11840, 12200, 757_760])
def test_gradients_norm_of_many_blocks(gdt, blocks):
    """Around the sizes at which the work is split in another way: tensors at odd places, a last block of one element.  The tolerance as above."""
    flat = _normal((256 * blocks + 64,), torch.float32, "many", blocks).to(DT[gdt])
    sizes, left, at, gs = [256 * 40, 256 * 7 + 1, 0, 255, 2, 256 * 500], blocks, 0, []
    left -= sum((n + 255) // 256 for n in sizes)
    for i, n in enumerate(sizes + [256 * (left - 1) + 1]):
        gs.append(flat[at + i: at + i + n])
        at += n
    plan = s2a.adamw_plan(None, gs, None, None)
    assert int(plan.plan.n_tensors) == len(gs) and sum((g.numel() + 255) // 256 for g in gs) == blocks
    clip = torch.full((2,), 9.0, device="cuda")
    scratch = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda").fill_(0xFF)
    s2a.s2a_grad_norm(plan, torch.tensor([0.0, 0.0, 1.0], device="cuda"), 2.0, clip, scratch)
    _done()
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in gs))
    assert abs(float(clip[0]) - norm) <= 8 * U * norm
    assert abs(float(clip[1]) - 2.0 / (norm + 1e-6)) <= 8 * U


def test_gradients_that_overflowed_change_nothing():
    for poison in (float("nan"), float("inf"), -float("inf")):
        ts = _tensors([1000, 30], torch.float32, torch.float32, 8, random.Random(1), "over", False)
        ts[1]["g"][7] = poison
        before = _clone(ts)
        plan = _plan(ts, 8, False)
        control, clip = torch.tensor([1e-3, 1.0, 1.0], device="cuda"), torch.empty(2, device="cuda")
        scratch = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda")
        s2a.s2a_grad_norm(plan, control, 1.0, clip, scratch)
        s2a.s2a_adamw_step(plan, control, clip=clip)
        _done()
        assert not math.isfinite(float(clip[0]))
        for b, a in zip(before, ts):
            for n in b:
                assert torch.equal(a[n].view(torch.uint8), b[n].view(torch.uint8))
        # without the clip's word the poison stays in its element, and in 8 bits in its block
        s2a.s2a_adamw_step(plan, control)
        _done()
        assert bool(torch.isfinite(ts[0]["p"]).all()) and int((~torch.isfinite(ts[1]["p"])).sum()) == 1


def test_zero_gradients_and_states():
    """All zeros stay zeros; the weights only decay; blocks of the smallest magnitudes become zeros, not NaN."""
    n = 700
    for bits in (32, 8):
        for tiny in (0.0, 1e-38, 1e-45):
            ts = _tensors([n], torch.float32, torch.float32, bits, random.Random(2), ("zero", bits), False)
            ts[0]["g"].fill_(tiny)
            for name in ("m", "v"):
                ts[0][name].view(torch.uint8).zero_()
                if bits == 8:
                    ts[0][name + "s"].zero_()
            p = ts[0]["p"].clone()
            plan = _plan(ts, bits, False, 0.5)
            s2a.s2a_adamw_step(plan, torch.tensor([0.1, 1.0, 1.0], device="cuda"), eps=1e-8)
            _done()
            want = p.double() * (1 - 0.1 * 0.5)
            assert torch.allclose(ts[0]["p"].double(), want, rtol=1e-6, atol=1e-20)
            assert bool(torch.isfinite(ts[0]["m"].float()).all()) and bool(torch.isfinite(ts[0]["v"].float()).all())


def test_a_small_root_keeps_a_code():
    """Beside a large one, a sqrt(v) far below the smallest code is stored as that code, not as zero."""
    for rng in (None, torch.tensor([5, 6], dtype=torch.int64, device="cuda")):
        ts = _tensors([512], torch.float32, torch.float32, 8, random.Random(3), "root", False)
        t = ts[0]
        for name in ("m", "v"):
            t[name].view(torch.uint8).zero_()
            t[name + "s"].zero_()
        t["g"].fill_(1e-9)
        t["g"][5] = 1e3
        t["g"][6] = 0.0
        s2a.s2a_adamw_step(_plan(ts, 8, False), torch.tensor([1e-3, 1.0, 1.0], device="cuda"), rng=rng)
        _done()
        codes = t["v"].view(torch.uint8)
        assert int(codes[5]) == 0x7E and int(codes[6]) == 0 and int(codes[7]) == 1 and int(codes[255]) == 1
        assert int(codes[300]) == 0x7E


def test_rounding_at_random_is_right_on_average():
    """A root that shrinks by 0.05 % a step stays where it is with nearest, and follows on average at random: the mean over 65536
    elements after 400 steps of v * 0.999 is within 4 % of 0.999^200 (a step's variance adds up to 6 % of v at most, half of
    it in the root), where nearest leaves 1."""
    n, steps = 65536, 400
    for random_bits in (False, True):
        ts = _tensors([n], torch.bfloat16, torch.float32, 8, random.Random(4), "mean", False)
        t = ts[0]
        t["m"].view(torch.uint8).zero_()
        t["g"].zero_()
        root = 0.3 + 0.4 * torch.rand(n, generator=_gen("roots"), device="cuda")
        root.view(-1, 256)[:, 0] = 1.0
        t["vs"].fill_(1.0)
        t["v"].copy_((root * 448).to(E4))
        start = t["v"].float().view(-1, 256)[:, 1:] / 448
        plan = _plan(ts, 8, False)
        control = torch.tensor([0.0, 1.0, 1.0], device="cuda")
        rng = torch.tensor([11, 0], dtype=torch.int64, device="cuda")
        for _ in range(steps):
            s2a.s2a_adamw_step(plan, control, rng=rng if random_bits else None)
            rng[1] += 1
        _done()
        now = t["v"].float().view(-1, 256) * (t["vs"] / 448)[:, None]
        # the first of each block holds the scale: it shrinks as the formula says in either way
        assert torch.allclose(now[:, 0], torch.full_like(now[:, 0], 0.999 ** (steps / 2)), rtol=1e-4)
        ratio = float((now[:, 1:] / start).mean())
        if random_bits:
            assert abs(ratio / 0.999 ** (steps / 2) - 1) < 0.04
        p = t["p"].clone()
    assert p.dtype is torch.bfloat16


def test_weights_rounded_at_random_move_on_average():
    """bfloat16 weights of 1 and an update of 1e-4, far below half their step of 2^-8: after 64 steps the mean has moved by
    64e-4 within 5 standard deviations of the sum (65536 elements, at most a step of 2^-8 each time)."""
    n = 65536
    p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(n, device="cuda")
    m, v = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    plan = s2a.adamw_plan([p], [g], [m], [v])
    control = torch.tensor([1e-4, 1e9, 1.0], device="cuda")
    rng = torch.tensor([3, 0], dtype=torch.int64, device="cuda")
    for _ in range(64):
        s2a.s2a_adamw_step(plan, control, rng=rng)
        rng[1] += 1
    _done()
    moved = 1 - float(p.double().mean())
    deviation = math.sqrt(64 * 1e-4 * 2.0 ** -8 / n)
    assert abs(moved - 64e-4) <= 5 * deviation + 64 * 1e-4 * 2.0 ** -7
    for _ in range(3):
        s2a.s2a_adamw_step(plan, control)      # to nearest nothing moves
    before = p.clone()
    s2a.s2a_adamw_step(plan, control)
    _done()
    assert torch.equal(p, before)


def test_replay_follows_its_control_and_other_streams():
    """A captured norm and step read learning rate, number and random words anew on every replay; the same as eager calls, bit for bit."""
    rng = random.Random(9)
    eager = _tensors([5000, 31, 1024], torch.bfloat16, torch.bfloat16, 8, rng, "replay", False)
    captured = _clone(eager)
    side = torch.cuda.Stream()

    def pieces(ts):
        plan = _plan(ts, 8, False, 0.1)
        return (plan, torch.tensor([1e-2, 1.0, 1.0], device="cuda"), torch.empty(2, device="cuda"),
                torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda"),
                torch.tensor([77, 5], dtype=torch.int64, device="cuda"))

    def call(plan, control, clip, scratch, words):
        s2a.s2a_grad_norm(plan, control, 0.5, clip, scratch)
        s2a.s2a_adamw_step(plan, control, clip=clip, rng=words, site=1)

    a, b = pieces(eager), pieces(captured)
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(*b)
    for i in range(3):
        for p in (a, b):
            p[1].copy_(torch.tensor([1e-2 / (i + 1), 1.0 + i, 1.0]))
            p[4][1] += 2
        torch.cuda.synchronize()
        call(*a)
        with torch.cuda.stream(side):
            graph.replay()
        _done()
        for x, y in zip(eager, captured):
            assert all(torch.equal(x[n].view(torch.uint8), y[n].view(torch.uint8)) for n in x)


def test_many_tensors_at_once():
    """3000 tensors of a few elements, one of them long."""
    sizes = [1 + i % 40 for i in range(3000)]
    sizes[1234] = 400_000
    ts = _tensors(sizes, torch.float32, torch.float32, 32, random.Random(5), "many", False, spread=0.3)
    before = _clone(ts)
    s2a.s2a_adamw_step(_plan(ts, 32, False), torch.tensor([1e-3, 2.0, 1.0], device="cuda"))
    _done()
    pick = [0, 1, 39, 40, 1233, 1234, 1235, 2999]
    hyper = (float(torch.tensor(1e-3)), 2.0, 1.0, 0.9, 0.999, 1e-8)
    _check_step([before[i] for i in pick], [ts[i] for i in pick], hyper, 32, [0.0] * 8, [1.0] * 8)
    for i, (a, b) in enumerate(zip(before, ts)):
        if i not in pick:
            assert not torch.equal(a["p"], b["p"])


class _Places(random.Random):
    """Offsets in the order given (a tensor takes its own, its gradient's, and one that is drawn between them)."""

    def __init__(self, places):
        super().__init__(8)
        self.places = list(places)

    def choice(self, among):
        return self.places.pop(0)


@pytest.mark.parametrize("pdt,gdt,bits,random_bits", [("bf16", "bf16", 8, True), ("f32", "bf16", 8, False), ("f32", "f32", 8, True),
                                                      ("f32", "bf16", 32, False), ("bf16", "bf16", 32, True)])
@pytest.mark.parametrize("blocks", [11_839, 11_840, 12_345, 757_759, 757_760])
def test_step_of_many_blocks(pdt, gdt, bits, random_bits, blocks):
    """On both sides of the sizes at which a warp takes more blocks at a time: tensors that begin and end inside of what it takes, on the
    16-byte grid and beside it."""
    ends = [1000, 256 * 1003 + 5, 300, 777]
    sizes = ends[:2] + [256 * (blocks - 1 - sum(-(-n // 256) for n in ends)) + 9] + ends[2:]
    assert sum(-(-n // 256) for n in sizes) == blocks
    copies = pdt == "f32"
    for beside in ((1, 2), (2, 4)) if blocks < 20_000 else ((1, 3),):   # the tensors that lie off the grid
        places = []
        for i in range(len(sizes)):
            at = 3 if i in beside else 0
            places += [at, 5, at]
        ts = _tensors(sizes, DT[pdt], DT[gdt], bits, _Places(places), (pdt, gdt, bits, blocks), copies)
        before = _clone(ts)
        hyper = (float(torch.tensor(1e-2)), 7.0, 0.25, 0.9, 0.999, 1e-8)
        draws = (77, 12)
        state = torch.tensor(draws, dtype=torch.int64, device="cuda") if random_bits else None
        s2a.s2a_adamw_step(_plan(ts, bits, copies, 0.1), torch.tensor(hyper[:3], device="cuda"), *hyper[3:], rng=state, site=3)
        _done()
        block0 = 0
        for b, a, n in zip(before, ts, sizes):
            long = 256 * 70
            for start in sorted({0, max(0, n // 512 * 256 - long), max(0, n - long) // 256 * 256}):
                stop = min(n, start + long + 256)
                rows = slice(start // 256, -(-stop // 256))
                part = [{name: t[name][rows] if name in ("ms", "vs") else t[name][start:stop] for name in t} for t in (b, a)]
                _check_step(part[:1], part[1:], hyper, bits, [0.1], [1.0], draws if random_bits else None, 3, pdt=DT[pdt],
                            block0=block0 + start // 256)
            moved = a["p"] != b["p"]
            # No block is left out: each update is some 1.6e-3 of its weight or more (the decay alone 1e-3), a fifth of a bfloat16 step at random, and 256
            # weights stay where they are once in 0.8^-256 = 1e24 blocks; binary32 weights of 1e-3 and more all move.
            assert bool(moved[: n // 256 * 256].view(-1, 256).any(1).all())
            block0 += -(-n // 256)


def test_beta_zero_and_betas_near_one():
    for b1, b2 in ((0.0, 0.0), (0.0, 0.999999), (0.9999, 0.5)):
        ts = _tensors([777], torch.float32, torch.float32, 32, random.Random(6), ("betas", b1), False)
        before = _clone(ts)
        s2a.s2a_adamw_step(_plan(ts, 32, False), torch.tensor([1e-3, 1.0, 1.0], device="cuda"), b1, b2, 1e-8)
        _done()
        _check_step(before, ts, (float(torch.tensor(1e-3)), 1.0, 1.0, b1, b2, 1e-8), 32, [0.0], [1.0])


def test_states_rounded_at_random_follow_where_nearest_stays():
    """Under a scale that stays 1 (the first element of each block has a state and a gradient of 1, the others none) m shrinks by 0.1 % a step and
    sqrt(v) by 0.05 %, far less than half a code's step.  To nearest, all codes stay.  At random a state's mean is the formula's:
    a code's step is at most 1/8 of its value, so that a step d (1e-3, 5e-4 of the value) adds a variance of at most d / 8, 400 steps 0.05
    and 0.025, of which the mean over 65280 elements has a deviation of 8.8e-4 and 6.2e-4; five of them, 400 times the half of a
    16-bit field's last place (2^-17 of 1/8: 3.9e-4), and 400 steps of the scale, each off by at most
    8 u (five roundings on the way to a, two of the sum of squares, half of them in the root, and one step of the root): 2e-4."""
    n, steps, b1, b2 = 65536, 400, 0.999, 0.999
    gen = _gen("follow")
    start = 0.3 + 0.4 * torch.rand(2, n, generator=gen, device="cuda")
    start[0] *= torch.where(torch.rand(n, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    start.view(2, -1, 256)[:, :, 0] = 1.0
    g = torch.zeros(n, device="cuda")
    g[::256] = 1.0
    for random_bits in (False, True):
        m, v = ((x * 448).to(E4) for x in start)
        scales = [torch.ones(n // 256, device="cuda") for _ in range(2)]
        first = [x.float().clone() for x in (m, v)]
        p = torch.zeros(n, device="cuda")
        plan = s2a.adamw_plan([p], [g], [m], [v], [scales[0]], [scales[1]])
        control = torch.tensor([0.0, 1.0, 1.0], device="cuda")
        rng = torch.tensor([11, 0], dtype=torch.int64, device="cuda")
        for _ in range(steps):
            s2a.s2a_adamw_step(plan, control, b1, b2, rng=rng if random_bits else None)
            rng[1] += 1
        _done()
        for x, s, was, kept, deviation in ((m, scales[0], first[0], b1 ** steps, 8.8e-4), (v, scales[1], first[1], b2 ** (steps / 2), 6.2e-4)):
            assert float((s - 1).abs().max()) <= 2e-4
            now = x.float()
            assert bool((now.view(-1, 256)[:, 0] == 448).all())
            if random_bits:
                ratio = (now * s.repeat_interleave(256) / was).view(-1, 256)[:, 1:]
                assert abs(float(ratio.double().mean()) - kept) <= 5 * deviation + 3.9e-4 + 2e-4
            else:
                assert torch.equal(now, was)


@pytest.mark.parametrize("gdt,random_bits", [("f32", False), ("f32", True), ("bf16", False), ("bf16", True)])
def test_8_bit_states_are_the_formulas_bit_for_bit(gdt, random_bits):
    """Four steps by elementary operations, each rounded to binary32: m + (1 - b1)(g' - m), b2 v + ((1 - b2) g') g', the root, the largest of a block,
    448 times its reciprocal, the product with that and the code.  No code and no scale differs; so none differs in the steps after."""
    n, b1, b2 = 40_000, 0.9, 0.999
    f = lambda x: torch.tensor(x, dtype=torch.float32, device="cuda")  # noqa: E731
    blocks = -(-n // 256)
    grow = 10 ** (20 * torch.rand(blocks, generator=_gen("grow"), device="cuda") - 12)       # a block's magnitudes, 1e-12 to 1e8
    per = lambda s: s.repeat_interleave(256)[:n]  # noqa: E731
    rows = lambda x: torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)  # noqa: E731
    g = (_normal((n,), torch.float32, "bits", gdt) * per(grow)).to(DT[gdt])
    g[1000:1300] = 0
    p = torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4) for _ in range(2))
    ms, vs = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
    plan = s2a.adamw_plan([p], [g], [m], [v], [ms], [vs])
    control = torch.tensor([1e-3, 0.0, 0.37], device="cuda")
    words = torch.tensor([123456789, 77], dtype=torch.int64, device="cuda")
    code_m, code_v, top_m, top_v = (t.clone() for t in (m, v, ms, vs))
    scaled = g.float() * control[2]
    for number in range(1, 5):
        control[1] = number
        words[1] += 1
        s2a.s2a_adamw_step(plan, control, b1, b2, rng=words if random_bits else None, site=5)
        o = code_m.float() * per(top_m * f(1 / 448))
        r = code_v.float() * per(top_v * f(1 / 448))
        want_m = o + f(1 - b1) * (scaled - o)
        root = (f(b2) * (r * r) + (f(1 - b2) * scaled) * scaled).double().sqrt().float()
        bits = _fields(n, 0, words.tolist(), 5, False) if random_bits else None
        codes = []
        for x, draws in ((want_m, bits), (root, None if bits is None else (bits % 256) * 256 + bits // 256)):
            top = rows(x.abs()).amax(1)
            codes.append(top)
            magnitude = x.abs() * per(torch.where(top > 0, (1 / top.double()).float() * 448, 0.0))
            if bits is None:
                codes.append(magnitude.to(E4).view(torch.uint8).int())
            else:
                codes.append((((magnitude * 2.0 ** -120).view(torch.int32) + ((draws.int() << 4) | 8)) >> 20).clamp(max=0x7E))
        top_m, code_m, top_v, code_v = codes
        code_m = (code_m | ((want_m < 0).int() << 7)).to(torch.uint8).view(E4)
        code_v = torch.where(root > 0, code_v.clamp(min=1), code_v).to(torch.uint8).view(E4)
        _done()
        assert torch.equal(ms, top_m) and torch.equal(vs, top_v)
        # (a code of zero may have either sign)
        assert torch.equal(m.float(), code_m.float()) and torch.equal(v.view(torch.uint8), code_v.view(torch.uint8))
    assert int((v.view(torch.uint8) == 0).sum()) == 300


def test_roots_beyond_the_range():
    """A finite gradient whose square is beyond binary32 leaves its weight (an update of m over an infinity) and the others; zeros and squares below the
    normal range have the root zero."""
    n = 512
    for random_bits in (False, True):
        p, g = torch.ones(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
        g[3], g[300], g[301] = 1e25, 0.0, 1e-22
        m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4) for _ in range(2))
        scales = [torch.zeros(n // 256, device="cuda") for _ in range(2)]
        words = torch.tensor([5, 6], dtype=torch.int64, device="cuda") if random_bits else None
        s2a.s2a_adamw_step(s2a.adamw_plan([p], [g], [m], [v], [scales[0]], [scales[1]]), torch.tensor([1e-2, 1.0, 1.0], device="cuda"), rng=words)
        _done()
        assert bool(torch.isfinite(p).all()) and float(p[3]) == 1.0 and float(p[300]) == 1.0 and bool((p[:3] < 1).all())
        assert float(scales[1][0]) == math.inf and math.isfinite(float(scales[1][1]))
        assert not v.view(torch.uint8)[300:302].any() and int((v.view(torch.uint8)[256:] == 0).sum()) == 2
