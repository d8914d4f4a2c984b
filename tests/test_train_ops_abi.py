"""Host-side checks of rotary positions, the norms of queries and keys, the AdamW step and the gradients' norm that need no GPU: refusals (all
before any launch), the overlap rules against a walk over every byte, the table of turns against whole numbers, and the plan of a step."""
import ctypes
import itertools
import math
import os
import random
import shutil
import subprocess
from fractions import Fraction

import pytest
import torch

from paper_2503_08154_b200 import binding, build

F32, BF16 = 0, 1
OK, NULL, SHAPE, ALIGN, DTYPE, CUDA, OVERLAP, VALUE = 0, 1, 2, 3, 4, 5, 8, 9
A, B, C, D, E, F, G = (0x10000000 * i for i in range(1, 8))   # far apart, never dereferenced
NO_GPU = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that pass every check would be launched on addresses that do not exist")

FIELDS = ("q k out_q out_k positions table gamma_q gamma_k grad_q grad_k grad_gamma_q grad_gamma_k scratch first "
          "scale eps interleaved dt wdt").split()
SIZES = "pos_batch pos_axis axes batch tokens heads_q heads_k head_dim rot_dim".split()
STRIDES = ("q_stride", "k_stride", "out_q_stride", "out_k_stride", "grad_q_stride", "grad_k_stride")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _args(**changes):
    v = dict(q=A, k=B, out_q=C, out_k=D, positions=E, table=F, gamma_q=E, gamma_k=E, grad_q=G, grad_k=G + 0x100000, grad_gamma_q=0,
             grad_gamma_k=0, scratch=0, first=0, pos_batch=8, pos_axis=0, axes=1, batch=2, tokens=8, heads_q=4, heads_k=2, head_dim=64, rot_dim=64,
             scale=1.0, eps=1e-6, interleaved=0, dt=BF16, wdt=F32)
    v |= {"q_stride": (8 * 256, 256, 64), "out_q_stride": (8 * 256, 256, 64), "grad_q_stride": (8 * 256, 256, 64)}
    v |= {"k_stride": (8 * 128, 128, 64), "out_k_stride": (8 * 128, 128, 64), "grad_k_stride": (8 * 128, 128, 64)}
    v |= changes
    return binding._rope_call(*(v[n] for n in FIELDS)) + binding._rope_sizes(*(v[n] for n in SIZES), *(s for n in STRIDES for s in v[n]))


CALLS = ("s2a_rope_fwd", "s2a_rope_bwd", "s2a_qknorm_rope_fwd", "s2a_qknorm_rope_bwd")


@pytest.mark.parametrize("name", CALLS)
def test_rope_refusals(lib, name):
    def call(**changes):
        return getattr(lib, name)(_args(**changes), None)

    norm, bwd = "qknorm" in name, name.endswith("rope_bwd") and "qknorm" in name
    assert getattr(lib, name)(None, None) == NULL
    for none in ({"batch": 0}, {"tokens": 0}, {"heads_q": 0, "heads_k": 0}):
        assert call(**none) == OK                                     # nothing to do
    assert call(dt=2) == DTYPE and call(dt=-1) == DTYPE
    for bad in ({"head_dim": 0}, {"head_dim": 513}, {"rot_dim": 63}, {"rot_dim": 66}, {"axes": 0}, {"axes": 5}, {"heads_q": 65536},
                {"batch": 1 << 31}, {"tokens": 1 << 31}, {"batch": 1 << 16, "tokens": 1 << 16}, {"pos_batch": 1 << 40}, {"pos_axis": 1 << 60},
                {"q_stride": (1 << 62, 256, 64)}, {"q_stride": (8 * 256, 256, 1 << 32)},
                {"out_q_stride": (8 * 256, 256, 63)}, {"out_q_stride": (0, 256, 64)}, {"out_k_stride": (1024, 0, 64)}, {"out_q_stride": (256, 256, 64)}):
        assert call(**bad) == SHAPE, bad
    for scale in (float("nan"), float("inf"), -float("inf")):
        assert call(scale=scale) == VALUE
    for missing in ("q", "k", "out_q", "out_k", "table"):
        assert call(**{missing: 0}) == NULL, missing
    assert call(positions=0, axes=2) == NULL
    for bad in ({"q": A + 1}, {"out_k": D + 1}, {"table": F + 8}, {"positions": E + 2}, {"dt": F32, "q": A + 2}):
        assert call(**bad) == ALIGN, bad
    # into the other tensor, and within the own one but not in place
    for bad in ({"out_q": A + 2}, {"out_q": A, "out_q_stride": (16 * 256, 256, 64)}, {"out_q": B + 64}, {"out_k": A + 128}, {"out_k": C + 128}):
        assert call(**bad) == OVERLAP, bad
    if norm:
        assert call(wdt=3) == DTYPE and call(gamma_q=E + 2) == ALIGN
        for eps in (-1.0, float("nan"), float("inf")):
            assert call(eps=eps) == VALUE
    else:
        assert call(rot_dim=0) == SHAPE
    if bwd:
        assert call(grad_q=0) == NULL and call(grad_k=0) == NULL and call(grad_gamma_q=E) == NULL       # sums need scratch
        assert call(grad_gamma_k=E, scratch=F + 8) == ALIGN and call(grad_gamma_q=E + 2, scratch=F) == ALIGN
        assert call(grad_q=G + 1) == ALIGN and call(out_q=G + 64) == OVERLAP
    assert binding.qknorm_rope_scratch_bytes(1, 1, 1, 1, 0) == 0 and binding.qknorm_rope_scratch_bytes(1, 1, 1, 1, 513) == 0
    assert binding.qknorm_rope_scratch_bytes(4, 5, 6, 7, 100) == 296 * 100 * 4


def _bytes(at, n, s, row):
    return {at + a * s[0] + b * s[1] + c * s[2] + i for a, b, c in itertools.product(*map(range, n)) for i in range(row)}


@NO_GPU
def test_overlap_rules_against_every_byte(lib):
    """Two tensors inside one buffer: what shares no byte is accepted where both step alike or lie apart, and what shares one never is."""
    rng = random.Random(0)
    refused = accepted = apart = 0
    for _ in range(700):
        n = (rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3))
        d = rng.choice([2, 4])
        heads_k = rng.randint(1, 3)

        def strides(heads):
            order = rng.choice([(0, 1, 2), (0, 2, 1), (1, 0, 2)])
            size, s, step = (n[0], n[1], heads), [0, 0, 0], d
            for i in reversed(order):
                s[i] = step
                step = step * size[i] + rng.choice([0, 0, d, 2 * d])
            return tuple(s)

        packed = rng.random() < 0.7                        # one buffer, the same steps
        sq = strides(n[2] + (heads_k if packed else 0))
        sk = sq if packed else strides(heads_k)
        gap = rng.choice([0, n[2] * sq[2], rng.randrange(0, 60)])
        q, k = A, A + 4 * gap
        status = lib.s2a_rope_fwd(_args(q=q, k=k, out_q=q, out_k=k, dt=F32, batch=n[0], tokens=n[1], heads_q=n[2], heads_k=heads_k, head_dim=d,
                                        rot_dim=d, q_stride=sq, out_q_stride=sq, k_stride=sk, out_k_stride=sk, positions=0), None)
        bq = _bytes(q, n, [4 * s for s in sq], 4 * d)
        bk = _bytes(k, (n[0], n[1], heads_k), [4 * s for s in sk], 4 * d)
        folded = len(bk) < n[0] * n[1] * heads_k * 4 * d or len(bq) < n[0] * n[1] * n[2] * 4 * d
        if folded:
            assert status == SHAPE
        elif bq & bk:
            refused += 1
            assert status == OVERLAP
        else:
            apart += 1
            accepted += status == CUDA                     # every check passed; there is no GPU to launch on
            assert status in (CUDA, OVERLAP)
            if packed and gap == n[2] * sq[2] and sq[2] == d:
                assert status == CUDA, (n, heads_k, sq)
    assert refused > 80 and apart > 80 and accepted > 0.7 * apart


def test_table_of_turns(lib):
    def table(*args, **kw):
        return [(a % (1 << 64), b) for a, b in binding.rope_table(*args, **kw).tolist()]

    # whole numbers where the power is one: base 16, pairs 0, 1, 2, 3 of 4 have the frequencies 1, 1/2, 1/4, 1/8
    turn = Fraction(1 << 64) / Fraction(2 * 3141592653589793238462643383279502884197, 10 ** 39)
    for got, want in zip(table(8, base=16.0), (turn, turn / 2, turn / 4, turn / 8)):
        assert abs(got[0] - want) <= 2 and got[1] == 0
    for (a, _), (b, _) in zip(table(64), table(64, scaling="linear", factor=4.0)):
        assert abs(a - 4 * b) <= 8
    first, last = table(64), table(64, scaling="base", factor=8.0)
    # entries are rounded to even numbers: off by 1 at most, which 8 multiplies
    assert abs(first[0][0] - last[0][0]) <= 2 and abs(first[-1][0] - 8 * last[-1][0]) <= 9 + first[-1][0] * 2.0 ** -50
    plain, parts = table(128), table(128, scaling="parts", factor=8.0, original_length=4096, slow=1.0, fast=32.0)
    for (a, _), (b, _) in zip(plain, parts):
        turns = 4096 * a / 2 ** 64
        keep = min(1.0, max(0.0, (turns - 1) / 31))
        assert abs(b - a * (keep + (1 - keep) / 8)) <= 2 + a * 2.0 ** -50
    axes = table(48, axes=3)
    assert [b for _, b in axes] == [0] * 8 + [1] * 8 + [2] * 8 and axes[:8] == [(a, 0) for a, _ in axes[16:]]
    assert table(0) == []
    buf = (ctypes.c_uint64 * 64)()

    def call(rot=16, base=1e4, scaling=0, factor=2.0, length=100.0, slow=1.0, fast=32.0, axes=1, out=buf):
        return lib.s2a_rope_table(out, rot, base, scaling, factor, length, slow, fast, axes)

    assert call() == OK and call(rot=15) == SHAPE and call(rot=514) == SHAPE and call(axes=0) == SHAPE and call(axes=3) == SHAPE and call(axes=5) == SHAPE
    assert call(out=None) == NULL
    for bad in ({"base": 0.5}, {"base": float("nan")}, {"base": float("inf")}, {"scaling": 4}, {"scaling": -1}, {"scaling": 1, "factor": 0.0},
                {"scaling": 2, "factor": float("inf")}, {"scaling": 3, "length": 0.0}, {"scaling": 3, "slow": 32.0}, {"scaling": 3, "slow": -1.0},
                {"scaling": 3, "fast": float("inf")}):
        assert call(**bad) == VALUE, bad
    with pytest.raises(binding.S2AError, match="scaling"):
        binding.rope_table(64, scaling="other")


def _tensor(i=0, n=1000, bits=32, copy=None, **changes):
    base = 0x100000000 * (i + 1)
    t = binding._StepTensor()
    t.param, t.grad, t.exp_avg, t.exp_avg_sq = (base + 0x10000000 * k for k in range(4))
    if bits == 8:
        t.exp_avg_scale, t.exp_avg_sq_scale = base + 0x40000000, base + 0x50000000
    t.copy = copy
    t.n, t.weight_decay, t.lr_scale = n, 0.1, 1.0
    for k, v in changes.items():
        setattr(t, k, v)
    return t


def _fill(lib, tensors, pdt=F32, gdt=F32, bits=32):
    records = (binding._StepTensor * max(1, len(tensors)))(*tensors)
    size = lib.s2a_step_plan_bytes(records, len(tensors))
    room = (ctypes.c_uint64 * (size // 8 + 4))()
    at = ctypes.addressof(room)
    plan = binding._StepPlan()
    status = lib.s2a_step_plan_fill(records, len(tensors), pdt, gdt, bits, at + -at % 16, ctypes.byref(plan))
    owner = (ctypes.c_uint32 * plan.n_chunks).from_buffer_copy(ctypes.string_at(at + -at % 16 + 96 * len(tensors), 4 * plan.n_chunks)) if status == OK else []
    return status, plan, size, list(owner)


def test_plan_of_a_step(lib):
    status, plan, size, owner = _fill(lib, [_tensor(0, 1), _tensor(1, 256), _tensor(2, 0), _tensor(3, 257)])
    assert status == OK and plan.bytes == size and plan.n_tensors == 4 and plan.chunk_blocks == 1 and owner == [0, 1, 3, 3]
    status, plan, size, owner = _fill(lib, [_tensor(0, 4_000_000), _tensor(1, 1)])
    assert status == OK and plan.chunk_blocks == 4 and owner == [0] * math.ceil(4_000_000 / 1024) + [1] and plan.bytes == size
    assert _fill(lib, [])[0] == OK
    for bits in (8, 32):
        for name in ("param", "grad", "exp_avg", "exp_avg_sq") + (("exp_avg_scale", "exp_avg_sq_scale") if bits == 8 else ()):
            assert _fill(lib, [_tensor(bits=bits), _tensor(1, bits=bits, **{name: None})], bits=bits)[0] == NULL, name
            assert _fill(lib, [_tensor(1, 0, bits=bits, **{name: None}), _tensor(bits=bits)], bits=bits)[0] == OK     # empty: not looked at
    assert _fill(lib, [_tensor(param=None)])[0] == OK and _fill(lib, [_tensor(param=None)])[1].grads_only == 1
    assert _fill(lib, [_tensor()], pdt=4)[0] == DTYPE and _fill(lib, [_tensor()], gdt=-1)[0] == DTYPE and _fill(lib, [_tensor()], bits=16)[0] == VALUE
    assert _fill(lib, [_tensor(copy=0x90000000)], pdt=BF16)[0] == DTYPE
    for bad in ({"param": 0x100000002}, {"grad": 0x110000001}, {"exp_avg": 0x120000002}, {"exp_avg_sq": 0x130000001}, {"copy": 0x90000001}):
        assert _fill(lib, [_tensor(**bad)])[0] == ALIGN, bad
    for bad in ({"weight_decay": -0.1}, {"weight_decay": float("nan")}, {"lr_scale": float("inf")}, {"lr_scale": -1.0}):
        assert _fill(lib, [_tensor(**bad)])[0] == VALUE, bad
    a, b = _tensor(0), _tensor(1)
    assert _fill(lib, [a, a])[0] == OVERLAP                              # the same tensor twice
    for name in ("param", "exp_avg", "exp_avg_sq"):
        assert _fill(lib, [a, _tensor(1, **{name: a.param + 3996})])[0] == OVERLAP
        assert _fill(lib, [a, _tensor(1, **{name: a.param + 4000})])[0] == OK
        assert _fill(lib, [a, _tensor(1, **{name: a.grad + 3996})])[0] == OVERLAP   # a gradient inside what is written
    assert _fill(lib, [a, _tensor(1, grad=a.grad)])[0] == OK             # shared gradients are only read
    assert _fill(lib, [a, b, _tensor(2, copy=b.exp_avg_sq + 8)])[0] == OVERLAP
    assert _fill(lib, [_tensor(bits=8), _tensor(1, bits=8, exp_avg_scale=0x140000000 + 12)], bits=8)[0] == OVERLAP
    assert lib.s2a_step_plan_bytes(None, 3) == 0


def test_step_and_norm_refusals(lib):
    _, plan, _, _ = _fill(lib, [_tensor()])
    p = ctypes.byref(plan)

    def step(plan=p, image=A, control=B, clip=None, rng=None, b1=0.9, b2=0.999, eps=1e-8):
        return lib.s2a_adamw_step(plan, image, control, clip, rng, 0, b1, b2, eps, None)

    assert step(plan=None) == NULL and step(image=None) == NULL and step(control=None) == NULL
    assert step(image=A + 8) == ALIGN and step(control=B + 2) == ALIGN and step(clip=C + 1) == ALIGN and step(rng=D + 4) == ALIGN
    for bad in ({"b1": 1.0}, {"b1": -0.1}, {"b2": 1.0}, {"b2": float("nan")}, {"eps": -1e-8}, {"eps": float("inf")}, {"eps": float("nan")}):
        assert step(**bad) == VALUE, bad
    _, grads, _, _ = _fill(lib, [_tensor(param=None)])
    assert step(plan=ctypes.byref(grads)) == NULL                       # gradients alone
    _, empty, _, _ = _fill(lib, [_tensor(n=0)])
    assert step(plan=ctypes.byref(empty), image=None) == OK

    def norm(plan=p, image=A, control=B, most=1.0, clip=C, scratch=D):
        return lib.s2a_grad_norm(plan, image, control, most, clip, scratch, None)

    assert norm(plan=None) == NULL and norm(image=None) == NULL and norm(control=None) == NULL and norm(clip=None) == NULL and norm(scratch=None) == NULL
    assert norm(most=-1.0) == VALUE and norm(most=float("nan")) == VALUE
    assert norm(scratch=D + 8) == ALIGN and norm(clip=C + 2) == ALIGN and norm(image=A + 4) == ALIGN
    assert lib.s2a_grad_norm_scratch_bytes(p) == 8 and lib.s2a_grad_norm_scratch_bytes(None) == 0


def test_struct_sizes_are_those_of_the_header(lib):
    # 13 pointers, 28 words, 5 of four bytes and their padding; 7 pointers, a size, two floats; four sizes and four ints
    assert len(_args()) == 8 * 41 + 24 and ctypes.sizeof(binding._StepTensor) == 72 and ctypes.sizeof(binding._StepPlan) == 48


def test_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros(1, 2, 3, 64)
    with pytest.raises(binding.S2AError, match="CUDA"):
        binding.s2a_rope_fwd(x, None, x, None, None, binding.rope_table(64))
    with pytest.raises(binding.S2AError, match="table"):
        binding.s2a_rope_fwd(x, None, x, None, None, None)
    with pytest.raises(binding.S2AError, match="CUDA"):
        binding.adamw_plan(None, [torch.zeros(3)], None, None)
    for lists in (([x], [x, x], [x], [x]), (None, [x], [x], None), ([x], [x], None, [x])):
        with pytest.raises(binding.S2AError):
            binding.adamw_plan(*lists)


@pytest.mark.parametrize("name", CALLS)
def test_in_place_is_of_the_own_input_alone(lib, name):
    """An output may be the input that it belongs to; where the same tensor is the other side's input too, that one would be read while it
    is written."""
    def call(**changes):
        same = {"heads_k": 4, "k_stride": (8 * 256, 256, 64), "out_k_stride": (8 * 256, 256, 64), "grad_k_stride": (8 * 256, 256, 64)}
        return getattr(lib, name)(_args(**same | changes), None)

    for same in ({"k": A, "out_q": A}, {"k": A, "out_k": A}, {"q": B, "out_k": B}, {"q": B, "out_q": B}):
        assert call(**same) == OVERLAP, same
    # one head each
    ones = {"heads_q": 1, "heads_k": 1} | {n: (8 * 64, 64, 64) for n in STRIDES}
    assert call(k=A, out_q=A, **ones) == OVERLAP and call(k=A, out_k=A, **ones) == OVERLAP
    if name == "s2a_qknorm_rope_bwd":
        for same in ({"grad_k": G, "out_q": G}, {"grad_k": G, "out_k": G}, {"grad_q": B, "out_q": B}, {"k": G, "out_q": G}):
            assert call(**same) == OVERLAP, same
    if not torch.cuda.is_available():       # what is allowed passes every check; there is no GPU to launch on
        for fine in ({"k": A}, {"out_q": A}, {"out_k": B}, {"out_q": A, "out_k": B}):
            assert call(**fine) == CUDA, fine
        if name == "s2a_qknorm_rope_bwd":
            for fine in ({"out_q": G}, {"out_k": G + 0x100000}, {"grad_q": A, "out_q": A}, {"grad_k": G, "k": A}, {"q": G, "grad_k": A, "out_q": G}):
                assert call(**fine) == CUDA, fine


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("swap", [(0, 1), (1, 2), (0, 2)])
def test_in_place_has_the_same_strides_in_every_dimension(lib, name, swap):
    """An output at its input's address with two dimensions of equal extent exchanged has the same rows, each where another one's was."""
    whole = (16 * 64, 4 * 64, 64)                                      # 4 sequences, tokens, heads
    swapped = list(whole)
    swapped[swap[0]], swapped[swap[1]] = whole[swap[1]], whole[swap[0]]

    def call(**changes):
        return getattr(lib, name)(_args(**{"batch": 4, "tokens": 4, "heads_q": 4, "heads_k": 4} | {n: whole for n in STRIDES} | changes), None)

    for t, at, grad in (("q", A, G), ("k", B, G + 0x100000)):
        assert call(**{"out_" + t: at, "out_%s_stride" % t: tuple(swapped)}) == OVERLAP
        assert call(**{"out_" + t: at, "%s_stride" % t: tuple(swapped)}) == OVERLAP
        if name == "s2a_qknorm_rope_bwd":
            assert call(**{"out_" + t: grad, "out_%s_stride" % t: tuple(swapped)}) == OVERLAP
        if not torch.cuda.is_available():
            both = {"%s_stride" % t: tuple(swapped), "out_%s_stride" % t: tuple(swapped)}
            assert call(**{"out_" + t: at}) == CUDA and call(**{"out_" + t: at} | both) == CUDA
            # a dimension of one has no stride
            assert call(**{"out_" + t: at, "batch": 1, "out_%s_stride" % t: (7, *whole[1:])}) == CUDA


def test_without_heads_of_a_kind_its_pointers_are_ignored(lib):
    """heads_k = 0 or heads_q = 0: nothing of that kind is looked at, its weights included; the gradient of its weights is an output of the call."""
    for name in ("s2a_qknorm_rope_fwd", "s2a_qknorm_rope_bwd"):
        for side in ("q", "k"):
            odd = {n + side: 3 for n in ("", "out_", "gamma_", "grad_")} | {"heads_" + side: 0}
            assert getattr(lib, name)(_args(**odd, batch=0), None) == OK
            assert getattr(lib, name)(_args(**odd, **{"heads_" + ("k" if side == "q" else "q"): 0}), None) == OK
            if not torch.cuda.is_available():
                assert getattr(lib, name)(_args(**odd), None) == CUDA      # passes every check
    assert lib.s2a_qknorm_rope_bwd(_args(heads_k=0, grad_gamma_k=E + 2, scratch=F), None) == ALIGN
    assert lib.s2a_qknorm_rope_bwd(_args(heads_k=0, grad_gamma_k=E), None) == NULL     # sums need scratch


def test_binding_refuses_missing_tensors():
    """None, or a list, where a tensor is needed: an S2AError as for every other refusal."""
    x, table = torch.zeros(1, 2, 3, 64), binding.rope_table(64)
    for missing in (None, [1.0, 2.0, 3.0]):
        for call in (lambda: binding.s2a_rope_fwd(missing, None, x, None, None, table), lambda: binding.s2a_rope_bwd(missing, None, x, None, None, table),
                     lambda: binding.s2a_qknorm_rope_fwd(missing, None, None, None, x, None, None, table, 1e-6),
                     lambda: binding.s2a_qknorm_rope_bwd(x, None, missing, None, None, None, x, None, None, None, None, None, table, 1e-6),
                     lambda: binding.s2a_adamw_step(missing, x), lambda: binding.s2a_grad_norm(missing, x, 1.0, x, x)):
            with pytest.raises(binding.S2AError):
                call()
    with pytest.raises(binding.S2AError, match="output"):       # (a call with tensors on a GPU comes here)
        binding._rope(None, x, None, None, None, None, table, 1.0, False, 0, 0)
    for name, n in (("control", 3), ("clip", 2)):
        with pytest.raises(binding.S2AError, match=name):
            binding._float_words(None, n, name)
    with pytest.raises(binding.S2AError, match="exp_avg"):
        binding._state_bits(None, x)


def test_a_plans_image_is_kept_for_every_stream_that_reads_it(monkeypatch):
    """The image is memory of the stream current when the plan was made; each other stream that runs the plan is recorded with it, once."""
    recorded = []

    class Image:
        def record_stream(self, stream):
            recorded.append(stream)

    plan = binding.AdamWPlan()
    plan.image, plan.streams, plan.pairs = Image(), {100}, []
    now = 100
    monkeypatch.setattr(binding, "_stream_on", lambda dev: now)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: ("stream", now, dev))
    for now in (100, 200, 200, 100, 300, 200, 300):
        assert binding._plan_stream(plan, 1) == now
    assert recorded == [("stream", 200, 1), ("stream", 300, 1)]


def test_gradients_norm_where_clusters_of_sixteen_do_not_fit(lib, tmp_path):
    """The library's own host code against a runtime of the test's: small plans take one launch of a cluster where the device has room for one,
    and otherwise (a part of a GPU) the two launches of the others.  The device is asked once."""
    here = os.path.dirname(os.path.abspath(__file__))
    out = str(tmp_path / "fake.so")
    nvcc = shutil.which(os.environ.get("NVCC", "nvcc"))
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-Wl,-z,defs", "-Wl,-Bsymbolic", "-I", include, os.path.join(here, "fake_runtime.cpp"),
                    os.path.join(build.OBJ, "s2a_adamw.o"), "-o", out], check=True, capture_output=True)
    run = ctypes.CDLL(out).run_grad_norm
    grids, asked = (ctypes.c_uint * 16)(), ctypes.c_int()

    def launches(device, clusters, dtype, chunks):
        n = run(device, clusters, dtype, chunks, grids, ctypes.byref(asked))
        return list(grids[:n]) if n >= 0 else n

    for dtype in (F32, BF16):
        for device, clusters in ((0, 9), (1, 0), (2, -1), (3, 1), (70, 0), (71, 2)):   # (70, 71: beyond the devices that answers are kept for)
            for chunks in (1, 240, 2048):
                want = [16] if clusters > 0 else [-(-chunks // 8), 1]
                for _ in range(2):
                    assert launches(device, clusters, dtype, chunks) == want, (device, chunks)
            assert launches(device, clusters, dtype, 2049) == [257, 1]
        assert asked.value == (4 + 2 * 6) * (1 + (dtype == BF16))


@NO_GPU
def test_overlap_of_any_strides(lib):
    """Inputs, gradients and outputs with strides of their own, in any order of the dimensions, 0 among the inputs': a call that passes writes no byte that it
    reads elsewhere, nor one byte twice."""
    rng = random.Random(1)
    passed = refused = 0
    for _ in range(3000):
        n, heads, d, bwd = (rng.randint(1, 4), rng.randint(1, 4)), (rng.randint(1, 3), rng.randint(0, 3)), rng.choice([2, 4]), rng.random() < 0.5

        def strides(h, zero):
            s, step = [0, 0, 0], d
            for i in rng.sample(range(3), 3):
                s[i], step = step, step * max(1, (*n, h)[i]) + rng.choice([0, 0, 0, d, 1])
            if zero and rng.random() < 0.3:
                s[rng.randrange(3)] = rng.choice([0, d, 1])
            return tuple(s)

        places, often = {}, strides(max(heads), False)
        for name in ("q", "k", "out_q", "out_k") + (("grad_q", "grad_k") if bwd else ()):
            at = rng.choice([A + 4 * rng.choice([0, d * heads[0], rng.randrange(400)]), A + 40000 * (len(places) + 1)] + [v[0] for v in places.values()])
            places[name] = (at, rng.choice([often, strides(heads[name[-1] == "k"], not name.startswith("out"))]))
        call = lib.s2a_qknorm_rope_bwd if bwd else lib.s2a_rope_fwd
        status = call(_args(dt=F32, batch=n[0], tokens=n[1], heads_q=heads[0], heads_k=heads[1], head_dim=d, rot_dim=d, positions=0,
                            **{k: v[0] for k, v in places.items()}, **{k + "_stride": v[1] for k, v in places.items()}), None)
        size = {name: (*n, heads[name[-1] == "k"]) for name in places}
        touched = {name: _bytes(at, size[name], [4 * x for x in s], 4 * d) for name, (at, s) in places.items()}
        same = {name: (at, *(x for x, e in zip(s, size[name]) if e > 1)) for name, (at, s) in places.items()}
        bad = False
        for out in ("out_q", "out_k"):
            bad = bad or len(touched[out]) < math.prod(size[out]) * 4 * d
            for name in places:
                own = name[-1] == out[-1] and not name.startswith("out") and same[name] == same[out]
                bad = bad or (name != out and not own and bool(touched[out] & touched[name]))
        assert not (bad and status == CUDA), (n, heads, d, places)
        passed, refused = passed + (status == CUDA), refused + (status in (OVERLAP, SHAPE))
    assert passed > 300 and refused > 300


def test_a_plan_whose_gradients_were_replaced_is_refused():
    """One pair of parameter and gradient a call, in turn: all of them replaced is seen at once, one of them within a round."""
    plan = binding.AdamWPlan()
    params = [torch.zeros(3, requires_grad=True) for _ in range(3)]
    for p in params:
        p.grad = torch.ones(3)
    plan.pairs, plan.turn = [(p, p.grad) for p in params], 0
    for _ in range(4):
        binding._plan_current(plan)
    params[1].grad.zero_()
    params[2].grad = params[2].grad.detach()        # the same memory
    for _ in range(3):
        binding._plan_current(plan)
    params[0].grad = None
    with pytest.raises(binding.S2AError, match="another"):
        for _ in range(3):
            binding._plan_current(plan)
    for p in params:
        p.grad = torch.ones(3)
    with pytest.raises(binding.S2AError, match="another"):
        binding._plan_current(plan)
