"""A training step around attention put together from the library's calls, and the calls where programs strain them: tensors beyond 2^31
elements, first calls of a process under capture, side by side on two streams, and refusals of the binding.  Tolerances as in
test_rope_qknorm_gpu.py and test_adamw_gpu.py."""
import math
import os
import subprocess
import sys

import pytest
import torch

import test_adamw_gpu as step
import test_rope_qknorm_gpu as rope
from paper_2503_08154_b200 import binding as s2a

pytestmark = pytest.mark.gpu

U = rope.U
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Attention:
    """Queries and keys of x by two projections, their norms and the rotation, scores, a position bias, softmax with its stash, and the loss
    sum(w * probabilities); every product by torch, everything between the products by the library.  Weights, their gradients and
    the states lie in lists as a training program keeps them."""

    B, T, H, HK, D, C = 3, 37, 4, 2, 32, 48

    def __init__(self):
        B, T, H, HK, D, C = self.B, self.T, self.H, self.HK, self.D, self.C
        new = lambda *shape, scale=1.0: rope._normal(shape, torch.float32, "attention", shape, scale, scale=scale)  # noqa: E731
        self.x, self.w = new(B, T, C), new(B, H, T, T, scale=0.01)
        self.params = [new(C, H * D, scale=0.2), new(C, HK * D, scale=0.2), 1 + new(D, scale=0.1), 1 + new(1, D, scale=0.2).view(D),
                       new(32, H, scale=0.3)]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.table = s2a.rope_table(D).cuda()
        self.positions = torch.arange(T, dtype=torch.int32, device="cuda")
        self.buckets = s2a.log_buckets(1 - T, 2 * T - 1, 32, 128, True).cuda()
        self.q, self.k = torch.empty(B, T, H, D, device="cuda"), torch.empty(B, T, HK, D, device="cuda")
        self.rq, self.rk, self.dq, self.dk = (torch.empty_like(t) for t in (self.q, self.k, self.q, self.k))
        n = B * H * T * T
        self.prob, self.dscores = torch.empty(B, H, T, T, device="cuda"), torch.empty(B, H, T, T, device="cuda")
        self.codes, self.meta = s2a.alloc_stash(n, T, "cuda")
        byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.scratch = byte(s2a.qknorm_rope_scratch_bytes(B, T, H, HK, D))
        self.bias_scratch = byte(s2a.relbias_scratch_bytes(B, H, T, T, 32))
        codes = lambda p: torch.zeros(p.shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
        scales = lambda p: torch.zeros(-(-p.numel() // 256), device="cuda")  # noqa: E731
        self.state = [[codes(p) for p in self.params], [codes(p) for p in self.params], [scales(p) for p in self.params],
                      [scales(p) for p in self.params]]
        self.plan = s2a.adamw_plan(self.params, self.grads, *self.state, weight_decay=[0.1, 0.1, 0.0, 0.0, 0.0])
        self.control = torch.tensor([1e-2, 0.0, 1.0], device="cuda")
        self.clip = torch.empty(2, device="cuda")
        self.norm_scratch = byte(s2a.grad_norm_scratch_bytes(self.plan))
        self.rng = torch.tensor([21, 0], dtype=torch.int64, device="cuda")

    def forward(self):
        B, T, H, HK, D = self.B, self.T, self.H, self.HK, self.D
        self.q.copy_((self.x @ self.params[0]).view(B, T, H, D))
        self.k.copy_((self.x @ self.params[1]).view(B, T, HK, D))
        s2a.s2a_qknorm_rope_fwd(self.q, self.k, self.params[2], self.params[3], self.rq, self.rk, self.positions, self.table, 1e-6)
        scores = torch.einsum("bthgd,bshd->bhgts", self.rq.view(B, T, HK, H // HK, D), self.rk).reshape(B, H, T, T) / math.sqrt(D)
        scores = scores.contiguous()
        s2a.s2a_relbias_fwd(scores, self.params[4], self.buckets, scores, B, H, T, T)
        s2a.s2a_softmax_fwd(scores, self.prob, self.codes, self.meta, T)

    def backward(self):
        B, T, H, HK, D = self.B, self.T, self.H, self.HK, self.D
        s2a.s2a_softmax_bwd(self.w, self.codes, self.meta, self.dscores, T)
        s2a.s2a_relbias_bwd(self.dscores, self.buckets, self.grads[4], self.bias_scratch, B, H, T, T)
        d = self.dscores.view(B, HK, H // HK, T, T) / math.sqrt(D)
        gq = torch.einsum("bhgts,bshd->bthgd", d, self.rk).reshape(B, T, H, D).contiguous()
        gk = torch.einsum("bhgts,bthgd->bshd", d, self.rq.view(B, T, HK, H // HK, D)).contiguous()
        s2a.s2a_qknorm_rope_bwd(gq, gk, self.q, self.k, self.params[2], self.params[3], self.dq, self.dk, self.grads[2], self.grads[3], self.scratch,
                                self.positions, self.table, 1e-6)
        x = self.x.view(-1, self.C)
        torch.matmul(x.t(), self.dq.view(-1, H * D), out=self.grads[0])
        torch.matmul(x.t(), self.dk.view(-1, HK * D), out=self.grads[1])

    def update(self):
        s2a.s2a_grad_norm(self.plan, self.control, 0.5, self.clip, self.norm_scratch)
        s2a.s2a_adamw_step(self.plan, self.control, clip=self.clip, rng=self.rng, site=7)


def test_training_step_around_attention():
    """Three steps.  The gradients of all weights against 64-bit automatic differentiation of the same scores (from the gradient of the scores that
    the 4-bit stash gives, which both take as it is): products of at most 111 terms and the tolerances of the norm's backward pass are
    below 1e-5 of the norm of each gradient.  The update against the formula, from the state before it."""
    torch.backends.cuda.matmul.allow_tf32 = False
    a = Attention()
    B, T, H, HK, D = a.B, a.T, a.H, a.HK, a.D
    for number in range(1, 4):
        a.control[1] = number
        a.rng[1] += 16
        a.forward()
        a.backward()
        rope._done()
        leaves = [p.double().requires_grad_() for p in a.params]
        angle = rope._angles(a.table, a.positions, B, T)

        def turned(w, gamma, heads):
            v = (a.x.double() @ w).view(B, T, heads, D)
            v = v * ((v * v).mean(-1, keepdim=True) + 1e-6) ** -0.5 * gamma
            return rope._turn(v, angle, 1.0, False)[0]

        q, k = turned(leaves[0], leaves[2], H), turned(leaves[1], leaves[3], HK)
        scores = torch.einsum("bthgd,bshd->bhgts", q.view(B, T, HK, H // HK, D), k).reshape(B, H, T, T) / math.sqrt(D)
        at = torch.arange(T, device="cuda")
        scores = scores + leaves[4][a.buckets.long()[at[None, :] - at[:, None] + T - 1]].permute(2, 0, 1)
        assert float((torch.softmax(scores.detach(), -1) - a.prob).abs().max()) <= 1e-4      # the probabilities of these scores
        for leaf, got in zip(torch.autograd.grad((scores * a.dscores.double()).sum(), leaves), a.grads):
            assert float((got.double() - leaf).norm()) <= 1e-5 * float(leaf.norm())
        before = [{"p": p.clone(), "g": g.clone(), "m": m.clone(), "v": v.clone(), "ms": ms.clone(), "vs": vs.clone()}
                  for p, g, m, v, ms, vs in zip(a.params, a.grads, *a.state)]
        a.update()
        rope._done()
        norm = math.sqrt(sum(float(g.double().square().sum()) for g in a.grads))
        assert abs(float(a.clip[0]) - norm) <= 1e-6 * norm
        after = [{"p": p, "m": m, "v": v, "ms": ms, "vs": vs} for p, m, v, ms, vs in zip(a.params, *a.state)]
        for t in before:
            for n in ("p", "g", "m", "v"):
                t[n] = t[n].reshape(-1)
        after = [{n: (v.reshape(-1) if n in "pmv" else v) for n, v in t.items()} for t in after]
        hyper = (float(a.control[0]), float(number), 1.0, 0.9, 0.999, 1e-8)
        step._check_step(before, after, hyper, 8, [0.1, 0.1, 0.0, 0.0, 0.0], [1.0] * 5, (21, 16 * number), 7, clip=float(a.clip[1]))


def test_captured_update_is_the_eager_one():
    """Norm's backward pass, gradients' norm and step in one graph, replayed; the same bits as calls."""
    one, two = Attention(), Attention()
    for a in (one, two):
        a.forward()
        a.backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    gq, gk = torch.randn_like(one.q), torch.randn_like(one.k)

    def tail(a):
        s2a.s2a_qknorm_rope_bwd(gq, gk, a.q, a.k, a.params[2], a.params[3], a.dq, a.dk, a.grads[2], a.grads[3], a.scratch, a.positions, a.table, 1e-6)
        a.update()

    with torch.cuda.graph(graph, stream=side):
        tail(two)
    for number in range(1, 4):
        for a in (one, two):
            a.control[1] = number
            a.rng[1] += 3
        torch.cuda.synchronize()
        tail(one)
        with torch.cuda.stream(side):
            graph.replay()
        rope._done()
        for p, r in zip(one.params + one.grads + sum(one.state, []), two.params + two.grads + sum(two.state, [])):
            assert torch.equal(p.view(torch.uint8), r.view(torch.uint8))


CAPTURE = """
import sys
sys.path.insert(0, %r)
import torch
from paper_2503_08154_b200 import binding as s2a
bf = torch.bfloat16
shapes = [((2, 70, 6, 64), 2, bf), ((3, 5, 3, 256), 3, torch.float32), ((2, 33, 1, 40), 1, bf), ((1, 9, 2, 30), 1, torch.float32)]
work = []
for shape, hk, dt in shapes:
    q, g = (torch.randn(shape, device="cuda").to(dt) for _ in range(2))
    k, gk = (torch.randn(*shape[:2], hk, shape[3], device="cuda").to(dt) for _ in range(2))
    t = s2a.rope_table(shape[3]).cuda()
    pos = torch.arange(shape[1], dtype=torch.int32, device="cuda")
    w = torch.randn(shape[3], device="cuda")
    out = [torch.empty_like(x) for x in (q, k, q, k, q, k)] + [torch.empty_like(w) for _ in range(2)]
    sc = torch.empty(s2a.qknorm_rope_scratch_bytes(*shape[:3], hk, shape[3]), dtype=torch.uint8, device="cuda")
    work.append((q, k, g, gk, t, pos, w, out, sc))
p, g = [torch.randn(5000, device="cuda"), torch.randn(3, device="cuda")], [torch.randn(5000, device="cuda"), torch.randn(3, device="cuda")]
start = [x.clone() for x in p]
m, v = [torch.zeros_like(x) for x in p], [torch.zeros_like(x) for x in p]
plan = s2a.adamw_plan(p, g, m, v)
control, clip = torch.tensor([1e-3, 1.0, 1.0], device="cuda"), torch.empty(2, device="cuda")
ns = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda")
def step():
    for q, k, g_, gk, t, pos, w, out, sc in work:
        s2a.s2a_rope_fwd(q, k, out[0], out[1], pos, t)
        s2a.s2a_qknorm_rope_fwd(q, k, w, w, out[2], out[3], pos, t, 1e-6)
        s2a.s2a_qknorm_rope_bwd(g_, gk, q, k, w, w, out[4], out[5], out[6], out[7], sc, pos, t, 1e-6)
    s2a.s2a_grad_norm(plan, control, 1.0, clip, ns)
    s2a.s2a_adamw_step(plan, control, clip=clip)
def results():
    return [o.clone() for x in work for o in x[7]] + [o.clone() for o in p + m + v] + [clip.clone()]
def restart():
    for x, y in zip(p, start):
        x.copy_(y)
    for x in m + v:
        x.zero_()
torch.cuda.synchronize()
stream = torch.cuda.Stream()
with torch.cuda.stream(stream):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):   # the library's first calls in this process
        step()
restart()
torch.cuda.synchronize()
graph.replay()
torch.cuda.synchronize()
got = results()
restart()
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, results()))
print("same")
"""


def test_first_calls_of_a_process_may_be_captured():
    r = subprocess.run([sys.executable, "-c", CAPTURE % ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


def test_rows_far_apart():
    """Batches and heads more than 2^31 elements from one another, in a buffer of 9.7 GB."""
    far = (1 << 31) + 4096
    buf = torch.empty(2 * far + (1 << 29), dtype=torch.bfloat16, device="cuda")
    table = s2a.rope_table(64).cuda()
    gamma = rope._normal((64,), torch.float32, "gamma")
    for strides in ((far, 64, 8192, 1), (64 * 5, 64, far, 1)):        # by batch, by head
        near = rope._normal((2, 5, 3, 64), torch.bfloat16, "far", strides[0])
        heads = 2 if strides[2] == far else 3
        near = near[:, :, :heads].contiguous()
        x = torch.as_strided(buf, near.shape, strides)
        x.copy_(near)
        y = torch.as_strided(buf, near.shape, strides, storage_offset=1 << 20)
        want = [torch.empty_like(near) for _ in range(2)]
        s2a.s2a_qknorm_rope_fwd(near, None, gamma, None, want[0], None, None, table, 1e-6)
        s2a.s2a_rope_bwd(near, None, want[1], None, None, table)
        s2a.s2a_qknorm_rope_fwd(x, None, gamma, None, y, None, None, table, 1e-6)
        rope._done()
        assert torch.equal(y, want[0])
        s2a.s2a_rope_bwd(x, None, x, None, None, table)
        rope._done()
        assert torch.equal(x, want[1])
    del buf


def test_more_than_two_to_the_31_weights():
    """One tensor of 2^31 + 777 bfloat16 weights with 8-bit states: its last elements, checked against a small tensor of the same values, and the norm."""
    n = (1 << 31) + 777
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    codes = [torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(-(-n // 256), device="cuda") for _ in range(2)]
    tail = 777 + 256 * 5
    values = rope._normal((tail,), torch.bfloat16, "tail")
    g[-tail:] = values
    g[12345] = 2.0
    plan = s2a.adamw_plan([p], [g], [codes[0]], [codes[1]], [scales[0]], [scales[1]])
    control, clip = torch.tensor([1e-2, 1.0, 1.0], device="cuda"), torch.empty(2, device="cuda")
    scratch = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda")
    s2a.s2a_grad_norm(plan, control, math.inf, clip, scratch)
    s2a.s2a_adamw_step(plan, control)
    q = torch.ones(tail, dtype=torch.bfloat16, device="cuda")
    small = [torch.zeros(tail, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    top = [torch.zeros(-(-tail // 256), device="cuda") for _ in range(2)]
    s2a.s2a_adamw_step(s2a.adamw_plan([q], [values], [small[0]], [small[1]], [top[0]], [top[1]]), control)
    rope._done()
    norm = math.sqrt(float(values.double().square().sum()) + 4.0)
    assert abs(float(clip[0]) - norm) <= 8 * U * norm and float(clip[1]) == 1.0
    assert torch.equal(p[-tail:], q) and all(torch.equal(a[-tail:].view(torch.uint8), b.view(torch.uint8)) for a, b in zip(codes, small))
    assert all(torch.equal(a[-top[0].numel():], b) for a, b in zip(scales, top))
    assert float(p[12345]) < 1.0 and int((p[:-tail] != 1).sum()) == 1


def test_two_streams_side_by_side():
    """The same plan's tensors stay on one stream; separate calls on two streams at once give what they give alone."""
    cases = [rope._normal((2, 400, 12, 64), torch.bfloat16, "two", i) for i in range(2)]
    table = s2a.rope_table(64).cuda()
    gamma = rope._normal((64,), torch.float32, "gamma")
    scratch = [torch.empty(s2a.qknorm_rope_scratch_bytes(2, 400, 12, 0, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(i):
        out, sums = torch.empty_like(cases[i]), torch.empty(64, device="cuda")
        s2a.s2a_qknorm_rope_bwd(cases[1 - i], None, cases[i], None, gamma, None, out, None, sums, None, scratch[i], None, table, 1e-6)
        return out, sums

    alone = [call(i) for i in range(2)]
    rope._done()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        both = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                both.append(call(i))
        rope._done()
        assert all(torch.equal(a, b) for x, y in zip(alone, both) for a, b in zip(x, y))


def test_binding_refusals():
    x, table = torch.zeros(2, 3, 4, 64, device="cuda"), s2a.rope_table(64).cuda()
    y = torch.empty_like(x)

    def bad(match, *args, call=s2a.s2a_rope_fwd, **kw):
        with pytest.raises(s2a.S2AError, match=match):
            call(*args, **kw)

    pos = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    bad("heads", x[0], None, y[0], None, None, table)
    bad("like what", x, None, y[:, :2], None, None, table)
    bad("like what", x, None, y.bfloat16(), None, None, table)
    bad("dtype", x.half(), None, y.half(), None, None, table)
    bad("contiguous", x.transpose(2, 3).contiguous().transpose(2, 3), None, y, None, None, table)
    bad("keys", x, x[:, :2], y, y[:, :2], None, table)
    bad("needed", x, x, y, None, None, table)
    bad("table", x, None, y, None, None, table.float())
    bad("positions", x, None, y, None, pos.long(), table)
    bad("positions", x, None, y, None, pos[:, :2], table)
    bad("positions", x, None, y, None, pos[:1].expand(5, 3), table)
    bad("positions of", x, None, y, None, torch.zeros(3, 2, dtype=torch.int32, device="cuda").t(), table)
    bad("SHAPE", x, None, y[:1].expand_as(x), None, pos, table)
    bad("SHAPE", x, None, y, None, pos.expand(5, 2, 3), table)
    bad("plain numbers", x, None, y, None, pos, table, scale="one")
    bad("VALUE", x, None, y, None, pos, table, scale=math.nan)
    bad("one device", x, None, y, None, pos.cpu(), table)
    bad("gamma_q", x, None, x[0, 0, 0, :63], None, y, None, pos, table, 1e-6, call=s2a.s2a_qknorm_rope_fwd)
    bad("one dtype", x, x, x[0, 0, 0], x[0, 0, 0].bfloat16(), y, y.clone(), pos, table, 1e-6, call=s2a.s2a_qknorm_rope_fwd)
    bad("scratch", x, None, x, None, None, None, y, None, torch.empty(64, device="cuda"), None, None, pos, table, 1e-6, call=s2a.s2a_qknorm_rope_bwd)
    p, g = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    m, v = torch.zeros_like(p), torch.zeros_like(p)
    plan = lambda *a, **kw: s2a.adamw_plan(*a, **kw)  # noqa: E731
    bad("one entry", [p, p], [g], [m], [v], call=plan)
    bad("one entry", [p], [g], [m], [v], weight_decay=[0.0, 0.0], call=plan)
    bad("right size", [p], [g], [m[:200]], [v], call=plan)
    bad("contiguous", [p], [torch.zeros(600, device="cuda")[::2]], [m], [v], call=plan)
    bad("exp_avg", [p], [g], [m.half()], [v], call=plan)
    bad("one dtype", [p, p.clone()], [g, g.bfloat16()], [m, m.clone()], [v, v.clone()], call=plan)
    bad("scales", [p], [g], [m.to(torch.float8_e4m3fn)], [v.to(torch.float8_e4m3fn)], call=plan)
    bad("OVERLAP", [p, p], [g, g], [m, m.clone()], [v, v.clone()], call=plan)
    bad("bfloat16", [p], [g], [m], [v], copies=[p.clone()], call=plan)
    good = plan([p], [g], [m], [v])
    bad("control", good, torch.zeros(2, device="cuda"), call=s2a.s2a_adamw_step)
    bad("rng", good, torch.zeros(3, device="cuda"), rng=torch.zeros(3, dtype=torch.int64, device="cuda"), call=s2a.s2a_adamw_step)
    bad("VALUE", good, torch.zeros(3, device="cuda"), 1.0, call=s2a.s2a_adamw_step)
    bad("NULL", plan(None, [g], None, None), torch.zeros(3, device="cuda"), call=s2a.s2a_adamw_step)
    bad("scratch", good, torch.zeros(3, device="cuda"), 1.0, torch.zeros(2, device="cuda"), None, call=s2a.s2a_grad_norm)
    rope._done()


def test_binding_refuses_missing_tensors():
    x, table = torch.zeros(2, 3, 4, 64, device="cuda"), s2a.rope_table(64).cuda()
    p, g, m, v = (torch.zeros(300, device="cuda") for _ in range(4))
    good, control = s2a.adamw_plan([p], [g], [m], [v]), torch.zeros(3, device="cuda")
    clip, scratch = torch.zeros(2, device="cuda"), torch.empty(s2a.grad_norm_scratch_bytes(good), dtype=torch.uint8, device="cuda")
    for match, call in (("output", lambda: s2a.s2a_rope_fwd(x, None, None, None, None, table)),
                        ("output", lambda: s2a.s2a_rope_bwd(x, None, None, None, None, table)),
                        ("output", lambda: s2a.s2a_qknorm_rope_fwd(x, None, None, None, None, None, None, table, 1e-6)),
                        ("output", lambda: s2a.s2a_qknorm_rope_bwd(x, None, x, None, None, None, None, None, None, None, None, None, table, 1e-6)),
                        ("CUDA", lambda: s2a.s2a_qknorm_rope_bwd(x, None, None, None, None, None, x, None, None, None, None, None, table, 1e-6)),
                        ("control", lambda: s2a.s2a_adamw_step(good, None)), ("CUDA", lambda: s2a.s2a_adamw_step(good, [1e-3, 1.0, 1.0])),
                        ("plan", lambda: s2a.s2a_adamw_step(None, control)), ("plan", lambda: s2a.s2a_grad_norm(None, control, 1.0, clip, scratch)),
                        ("control", lambda: s2a.s2a_grad_norm(good, None, 1.0, clip, scratch)),
                        ("clip", lambda: s2a.s2a_grad_norm(good, control, 1.0, None, scratch)),
                        ("exp_avg", lambda: s2a.adamw_plan([p], [g], [None], [v]))):
        with pytest.raises(s2a.S2AError, match=match):
            call()
    rope._done()


def test_a_plan_may_be_dropped_while_another_stream_reads_it():
    """A plan of the current stream, run by a side stream that is busy, and dropped: its image's memory goes to nobody before the side stream has
    read it."""
    def tensors():
        return [rope._normal((n,), torch.float32, "dropped", n, i) for n in (3000, 17, 40_000) for i in range(2)]

    p, g = tensors(), [t * 0.1 for t in tensors()]
    q = [t.clone() for t in p]
    states = [[torch.zeros_like(t) for t in p] for _ in range(4)]
    control = torch.tensor([1e-2, 1.0, 1.0], device="cuda")
    clips = [torch.empty(2, device="cuda") for _ in range(2)]
    plan = s2a.adamw_plan(q, g, states[2], states[3])
    scratch = [torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda") for _ in range(2)]
    s2a.s2a_grad_norm(plan, control, 0.5, clips[1], scratch[1])
    s2a.s2a_adamw_step(plan, control, clip=clips[1])
    plan = s2a.adamw_plan(p, g, states[0], states[1])
    torch.cuda.synchronize()
    at, size = plan.image.data_ptr(), plan.image.numel() * 8
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                     # some 0.2 s
        s2a.s2a_grad_norm(plan, control, 0.5, clips[0], scratch[0])
        s2a.s2a_adamw_step(plan, control, clip=clips[0])
    del plan
    others = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(8)]
    busy = not side.query()
    places = [t.data_ptr() for t in others]
    rope._done()
    assert not busy or all(x + size <= at or at + size <= x for x in places)
    assert torch.equal(clips[0], clips[1])
    for a, b in zip(p + states[0] + states[1], q + states[2] + states[3]):
        assert torch.equal(a, b)


def test_training_with_gradients_that_stay():
    """Gradients of automatic differentiation that are zeroed in place stay where they are, and one plan serves all steps; with replaced ones (set to
    None) the old plan is refused, in place of a step with the old gradients, and a new one is right."""
    torch.backends.cuda.matmul.allow_tf32 = False
    sizes = [(40, 24), (24,), (24, 7)]
    params = [rope._normal(s, torch.float32, "stay", s, scale=0.3).requires_grad_() for s in sizes]
    x, w = rope._normal((50, 40), torch.float32, "x"), rope._normal((50, 7), torch.float32, "w", scale=0.1)
    states = [[torch.zeros(s, device="cuda") for s in sizes] for _ in range(2)]
    control = torch.tensor([1e-2, 0.0, 1.0], device="cuda")

    def backward():
        ((torch.tanh(x @ params[0] + params[1]) @ params[2]) * w).sum().backward()

    def update(number, plan):
        """The step, checked against the formula with the gradients that the parameters have now."""
        control[1] = number
        before = [{"p": p.detach().clone(), "g": p.grad.clone(), "m": m.clone(), "v": v.clone()} for p, m, v in zip(params, *states)]
        s2a.s2a_adamw_step(plan, control)
        rope._done()
        after = [{"p": p.detach(), "m": m, "v": v} for p, m, v in zip(params, *states)]
        flat = lambda ts: [{n: t.reshape(-1) for n, t in d.items()} for d in ts]  # noqa: E731
        step._check_step(flat(before), flat(after), (float(control[0]), float(number), 1.0, 0.9, 0.999, 1e-8), 32, [0.1] * 3, [1.0] * 3)

    def make():
        return s2a.adamw_plan(params, [p.grad for p in params], *states, weight_decay=0.1)

    backward()
    plan, places = make(), [p.grad.data_ptr() for p in params]
    update(1, plan)
    for number in (2, 3, 4):
        for p in params:
            p.grad.zero_()                      # optimizer.zero_grad(set_to_none=False)
        backward()
        assert [p.grad.data_ptr() for p in params] == places
        update(number, plan)
    for p in params:
        p.grad = None                           # optimizer.zero_grad()
    scratch, clip = torch.empty(s2a.grad_norm_scratch_bytes(plan), dtype=torch.uint8, device="cuda"), torch.empty(2, device="cuda")
    for again in (False, True):                 # nothing in their place yet, and others
        was = [t.detach().clone() for t in params + states[0] + states[1]]
        with pytest.raises(s2a.S2AError, match="another"):
            s2a.s2a_adamw_step(plan, control)
        with pytest.raises(s2a.S2AError, match="another"):
            s2a.s2a_grad_norm(plan, control, 1.0, clip, scratch)
        rope._done()
        assert all(torch.equal(a, b) for a, b in zip(was, params + states[0] + states[1]))
        backward()
    for p in params:
        p.grad = None
    backward()
    update(5, make())
