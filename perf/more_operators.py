"""What a training step or a decoding step runs around the scores and after the backward pass: rotary positions, the norms of
queries and keys with the rotation in the same pass, the AdamW step over many tensors, and the norm of all gradients.

Every operator has its plain form here (elementary torch operations in 32 bits, 64 for angles and long sums) beside the call
that a user makes of this repository's kernels (``own`` is true).

* rope: pairs of a head's first `rot` elements turn by position * frequency, (x, y) -> (x cos - y sin, x sin + y cos); a pair
  is (i, i + rot / 2) or (2 i, 2 i + 1); the elements beyond `rot` stay.  Cosine and sine are multiplied by `scale`.  The
  backward pass turns by the opposite angle.  With two axes the first half of the pairs goes by a token's row, the second by
  its column.  Scaled for long contexts: "linear" divides all frequencies by `factor`, "parts" those that turn less than
  once over the original length, and in part those up to 32 turns.
* qknorm: y = rope(x / sqrt(mean(x^2) + eps) * gamma) for each head's row.  Backward, from x alone: u = the gradient turned
  back, a = u * gamma, xhat = x * rstd, grad_x = rstd * (a - xhat * mean(a * xhat)), grad_gamma = sum of u * xhat.
* adamw: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) +
  eps).  In 8 bits the states are e4m3 codes of m and of sqrt(v), 448 standing for the largest magnitude of 256 elements,
  which is kept beside them in 32 bits; a sqrt(v) above zero has a code above zero.  Rounded to nearest, or at random: the
  bits below the last kept one get 16 bits of Philox4x32-10 added (Salmon et al., "Parallel random numbers: as easy as 1,
  2, 3", 2011).  Every tensor starts at a multiple of 256 in the count of elements that the random bits go by.
* gradnorm: norm = scale * sqrt(sum of g^2 over all tensors) and factor = min(1, max_norm / (norm + 1e-6)).
"""
import functools
import math

import torch

own = False

EPS = 1e-6
BETA1, BETA2, ADAM_EPS = 0.9, 0.999, 1e-8
MAX_NORM = 1.0
BLOCK = 256
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token for each of 64 sequences, at positions far into a long context; latency is all that counts
        {"name": "rope_fwd_one_token", "op": "rope", "pass": "fwd", "dtype": "bf16", "batch": 64, "tokens": 1, "heads_q": 32,
         "heads_k": 8, "head_dim": 128, "rot": 128, "interleaved": False, "axes": 1, "scaling": "parts", "layout": "packed"},
        # a long prompt, keys shared by four queries' heads
        {"name": "rope_fwd_long", "op": "rope", "pass": "fwd", "dtype": "bf16", "batch": 2, "tokens": 16384, "heads_q": 32,
         "heads_k": 8, "head_dim": 128, "rot": 128, "interleaved": False, "axes": 1, "scaling": "linear", "layout": "packed"},
        # gradients in float32, adjacent pairs, half of a head of 80 elements turned, an odd length
        {"name": "rope_bwd_part_odd_f32", "op": "rope", "pass": "bwd", "dtype": "f32", "batch": 3, "tokens": 2001, "heads_q": 16,
         "heads_k": 16, "head_dim": 80, "rot": 40, "interleaved": True, "axes": 1, "scaling": "none", "layout": "heads_first"},
        # queries and keys of a ViT-B/16 block, batch 64: patches go by row and column, queries and keys inside one buffer
        {"name": "qknorm_fwd_vit_b", "op": "qknorm", "pass": "fwd", "dtype": "bf16", "weights": "f32", "batch": 64,
         "tokens": 197, "heads_q": 12, "heads_k": 12, "head_dim": 64, "rot": 64, "interleaved": False, "axes": 2,
         "scaling": "none", "layout": "packed"},
        # the same in the backward pass, with the weights' gradients
        {"name": "qknorm_bwd_vit_b", "op": "qknorm", "pass": "bwd", "dtype": "bf16", "weights": "f32", "batch": 64,
         "tokens": 197, "heads_q": 12, "heads_k": 12, "head_dim": 64, "rot": 64, "interleaved": False, "axes": 2,
         "scaling": "none", "layout": "packed"},
        # the backward pass over long sequences with shared keys
        {"name": "qknorm_bwd_long", "op": "qknorm", "pass": "bwd", "dtype": "bf16", "weights": "bf16", "batch": 4,
         "tokens": 4097, "heads_q": 32, "heads_k": 8, "head_dim": 128, "rot": 128, "interleaved": False, "axes": 1,
         "scaling": "none", "layout": "packed"},
        # what a fine-tuning run with low-rank prompts trains: many small tensors
        {"name": "adamw32_prompts", "op": "adamw", "param": "f32", "grad": "f32", "states": 32, "random": False, "copies": False,
         "tensors": "prompts", "width": 1024, "blocks": 24, "ragged": False},
        # float32 weights with the bfloat16 copies that the next forward pass reads, 300 million of them
        {"name": "adamw32_copies_large", "op": "adamw", "param": "f32", "grad": "bf16", "states": 32, "random": False,
         "copies": True, "tensors": "blocks", "width": 1024, "blocks": 24, "ragged": False},
        # bfloat16 weights, states in 8 bits, everything rounded at random: 10 bytes an element instead of 28
        {"name": "adamw8_random_large", "op": "adamw", "param": "bf16", "grad": "bf16", "states": 8, "random": True,
         "copies": False, "tensors": "blocks", "width": 1024, "blocks": 24, "ragged": False},
        # tensors back to back at odd places of one buffer
        {"name": "adamw32_ragged", "op": "adamw", "param": "f32", "grad": "f32", "states": 32, "random": False, "copies": False,
         "tensors": "odd", "width": 257, "blocks": 40, "ragged": True},
        # the clip factor of a small and of a large model
        {"name": "gradnorm_prompts", "op": "gradnorm", "grad": "f32", "tensors": "prompts", "width": 1024, "blocks": 24,
         "ragged": False},
        {"name": "gradnorm_large", "op": "gradnorm", "grad": "bf16", "tensors": "blocks", "width": 1024, "blocks": 24,
         "ragged": False},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["rope", "rope", "qknorm", "qknorm", "adamw", "adamw", "gradnorm"])
    case = {"op": op}
    if op in ("rope", "qknorm"):
        head_dim = rng.choice([16, 32, 40, 64, 64, 72, 80, 96, 128, 128, 160, 192, 256, 2 * rng.randint(4, 128)])
        rot = head_dim if rng.random() < 0.6 else max(4, head_dim * rng.choice([1, 2, 3]) // 4 // 4 * 4)
        heads_q = rng.choice([1, 2, 3, 6, 8, 12, 16, 25, 32])
        heads_k = rng.choice([heads_q, heads_q, max(1, heads_q // 4), 1])
        most = (1 << 26) // ((heads_q + heads_k) * head_dim)
        tokens = rng.choice([1, _log_int(rng, 1, min(16384, most)), _log_int(rng, 2, min(16384, most))])
        case |= {"pass": rng.choice(["fwd", "bwd"]), "dtype": rng.choice(["bf16", "bf16", "f32"]), "tokens": tokens,
                 "batch": _log_int(rng, 1, max(1, min(256, most // tokens))), "heads_q": heads_q, "heads_k": heads_k,
                 "head_dim": head_dim, "rot": rot, "interleaved": rng.random() < 0.4,
                 "axes": 2 if rot % 4 == 0 and rng.random() < 0.25 else 1,
                 "scaling": rng.choice(["none", "linear", "parts"]), "layout": rng.choice(["packed", "heads_first", "separate"])}
        if op == "qknorm":
            case["weights"] = rng.choice(["bf16", "f32"])
        return case
    tensors = rng.choice(["prompts", "blocks", "odd"])
    width = _log_int(rng, 24, 1024)
    if tensors != "odd":
        width = max(24, width // 8 * 8)
    each = {"prompts": 14 * width, "blocks": 12 * width * width, "odd": 4 * width * width}[tensors]
    case |= {"grad": rng.choice(["bf16", "f32"]), "tensors": tensors, "width": width,
             "blocks": _log_int(rng, 1, max(1, min(48, 150_000_000 // each))), "ragged": False}
    if op == "gradnorm":
        return case | {"ragged": rng.random() < 0.3}
    states = rng.choice([8, 32])
    param = rng.choice(["bf16", "f32"])
    case |= {"param": param, "states": states, "random": rng.random() < 0.5, "copies": param == "f32" and rng.random() < 0.4}
    if states == 32 and not case["random"]:
        case["ragged"] = rng.random() < 0.3
    return case


def _sizes(case):
    """The lengths of the tensors of a step, in the order of their places."""
    w = case["width"]
    if case["tensors"] == "prompts":        # two factors of a prompt, two norms and four biases a block
        one = [197 * 8, 8 * w, w, w, w, w, w, w, w, 4 * w]
    elif case["tensors"] == "blocks":       # norms, query, key, value and output, then the two of the wider layer, with biases
        one = [w, w] + [w * w, w] * 4 + [w, w, 4 * w * w, 4 * w, 4 * w * w, w]
    else:
        one = [w, 3 * w * w + 1, 5, w * w + 2 * w + 3, 1]
    return one * case["blocks"]


def _places(case):
    """(sizes, starts, length of the buffer): starts are multiples of 256, or the tensors lie back to back."""
    sizes, starts, at = _sizes(case), [], 3 if case["ragged"] else 0
    for n in sizes:
        starts.append(at)
        at += n if case["ragged"] else -(-n // BLOCK) * BLOCK
    return sizes, starts, at


def work(case):
    if case["op"] in ("rope", "qknorm"):
        s = SIZE[case["dtype"]]
        tokens = case["batch"] * case["tokens"]
        n = tokens * (case["heads_q"] + case["heads_k"]) * case["head_dim"]
        small = 4 * tokens * case["axes"]
        if case["op"] == "rope":
            return {"bytes": 2 * n * s + small, "flops": 3 * n}
        weights = 2 * case["head_dim"] * SIZE[case["weights"]]
        if case["pass"] == "fwd":
            return {"bytes": 2 * n * s + small + weights, "flops": 7 * n}
        return {"bytes": 3 * n * s + small + 2 * weights, "flops": 16 * n}
    n = sum(_sizes(case))
    if case["op"] == "gradnorm":
        return {"bytes": n * SIZE[case["grad"]] + 8, "flops": 2 * n}
    each = 2 * SIZE[case["param"]] + SIZE[case["grad"]] + (16 if case["states"] == 32 else 4) + (2 if case["copies"] else 0)
    return {"bytes": n * each + (0 if case["states"] == 32 else 16 * (n // BLOCK)), "flops": 14 * n}


# ------------------------------------------------------------------------------------------ inputs
ORIGINAL, FACTOR, BASE = 8192, 16.0, 10000.0


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, scale=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0, scale, generator=gen).to(dtype)


def _heads(case, gen, heads, scale, first, width):
    """[batch, tokens, heads, head_dim] in the case's layout; `first` of `width` heads where queries and keys share a buffer."""
    b, t, d, dt = case["batch"], case["tokens"], case["head_dim"], DTYPES[case["dtype"]]
    values = _normal(gen, (b, t, heads, d), scale, dt)
    if case["layout"] == "heads_first":
        return values.transpose(1, 2).contiguous().transpose(1, 2)
    if case["layout"] == "packed":
        return torch.zeros((b, t, width, d), dtype=dt, device="cuda")[:, :, first:first + heads].copy_(values)
    return values


def _attention_inputs(case, seed):
    gen = _generator(seed)
    b, t, hq, hk, d, dt = (case[k] for k in ("batch", "tokens", "heads_q", "heads_k", "head_dim", "dtype"))
    state = {"case": case}
    if case["axes"] == 2:                   # patches of a window in rows, behind a class token
        side = max(1, math.isqrt(max(1, t - 1)))
        at = (torch.arange(t, device="cuda") - 1).clamp(min=0)
        state["positions"] = torch.stack([at // side, at % side])[:, None].expand(2, b, t).to(torch.int32).contiguous()
    else:                                   # a sequence each, whose tokens start anywhere in the context
        start = torch.randint(0, 120_000 if case["scaling"] != "none" else 4000, (b, 1), device="cuda", generator=gen)
        state["positions"] = (start + torch.arange(t, device="cuda")).to(torch.int32)
    state["scale"] = 1 + 0.1 * math.log(FACTOR) if case["scaling"] == "parts" else 1.0
    width = hq + 2 * hk                     # queries, keys and values side by side
    scale = 1.0 if case["pass"] == "fwd" or case["op"] == "qknorm" else 0.01
    state["q"] = _heads(case, gen, hq, scale, 0, width)
    state["k"] = _heads(case, gen, hk, scale, hq, width)
    for name in ("q", "k"):
        state["out_" + name] = torch.empty(state[name].shape, dtype=DTYPES[dt], device="cuda")
    if case["op"] == "qknorm":
        wt = DTYPES[case["weights"]]
        for name in ("q", "k"):
            state[name] *= 0.5 + 2 * torch.rand((1, 1, 1, d), device="cuda", generator=gen).to(DTYPES[dt])
            state["gamma_" + name] = (1 + _normal(gen, (d,), 0.3)).to(wt)
            if case["pass"] == "bwd":
                state["g_" + name] = _normal(gen, state[name].shape, 0.01, DTYPES[dt])
                state["grad_gamma_" + name] = torch.empty(d, dtype=wt, device="cuda")
    return state


def _views(flat, sizes, starts):
    return [flat[at:at + n] for n, at in zip(sizes, starts)]


def _step_inputs(case, seed):
    gen = _generator(seed)
    sizes, starts, total = _places(case)
    state = {"case": case, "sizes": sizes, "starts": starts,
             "control": torch.tensor([1e-3, 100.0 + seed % 57, 0.5], dtype=torch.float32, device="cuda")}   # lr, step, scale
    lengths = torch.tensor([b - a for a, b in zip(starts, starts[1:] + [total])], device="cuda")   # up to the next one's start
    # each tensor's gradients have their own magnitude; nothing lies between the tensors
    spread = torch.exp(torch.empty(len(sizes), device="cuda").normal_(-6, 1, generator=gen))
    inside = torch.zeros(total, dtype=torch.int8, device="cuda")
    for view in _views(inside, sizes, starts):
        view.fill_(1)
    grow = torch.repeat_interleave(spread, lengths, output_size=total - starts[0])
    grow = torch.nn.functional.pad(grow, (starts[0], 0)) * inside
    g = _normal(gen, (total,)).mul_(grow)
    state["g"] = (g * 2).to(DTYPES[case["grad"]])
    if case["op"] == "gradnorm":
        state["clip"] = torch.empty(2, dtype=torch.float32, device="cuda")
        return state
    state["p"] = (_normal(gen, (total,), 0.02) * inside).to(DTYPES[case["param"]])
    m = 0.3 * _normal(gen, (total,)).mul_(grow)
    r = (_normal(gen, (total,)).square_() + 0.05).sqrt_().mul_(grow)          # sqrt(v)
    if case["states"] == 32:
        state |= {"m": m, "v": r * r}
    else:
        for name, x in (("m", m), ("v", r)):
            rows = x.view(-1, BLOCK)
            largest = rows.abs().amax(dim=1, keepdim=True)
            state[name + "_scale"] = largest.view(-1).contiguous()
            state[name] = torch.where(largest > 0, rows * (448 / largest.clamp(min=1e-30)), 0.0).to(torch.float8_e4m3fn).view(-1)
    state["decay"] = [0.05 if n > 4 * case["width"] else 0.0 for n in sizes]   # none for norms and biases
    state |= {"decays": torch.tensor(state["decay"], device="cuda"), "lengths": lengths}
    if case["copies"]:
        state["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    if case["random"]:
        state["rng"] = torch.tensor([(seed * 0x9E3779B97F4A7C15 + 0x7654321) % (1 << 63), 5000 + seed % 911],
                                    dtype=torch.int64, device="cuda")
        state["site"] = 2 + seed % 5
    return state


def prepare(case, seed):
    return _attention_inputs(case, seed) if case["op"] in ("rope", "qknorm") else _step_inputs(case, seed)


# ------------------------------------------------------------------------------------------ plain forms
def _frequencies(case):
    """Radians a position for each pair, in 64 bits."""
    each = case["rot"] // 2 // case["axes"]
    w = BASE ** (-torch.arange(each, dtype=torch.float64, device="cuda") / each)
    if case["scaling"] == "linear":
        w = w / FACTOR
    elif case["scaling"] == "parts":
        keep = ((ORIGINAL * w / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        w = w / FACTOR * (1 - keep) + w * keep
    return w.repeat(case["axes"])


def _cos_sin(s, back):
    """[batch, tokens, 1, pairs] in 32 bits, from angles in 64."""
    c, w = s["case"], _frequencies(s["case"])
    if c["axes"] == 2:
        p = s["positions"].double()
        half = w.numel() // 2
        angle = torch.cat([p[0][..., None] * w[:half], p[1][..., None] * w[half:]], dim=-1)
    else:
        angle = s["positions"].double()[..., None] * w
    angle = angle[:, :, None] * (-1 if back else 1)
    return (torch.cos(angle) * s["scale"]).float(), (torch.sin(angle) * s["scale"]).float()


def _turn(x, cos, sin, rot, interleaved):
    """x in 32 bits."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, v], dim=-1).flatten(-2) if interleaved else torch.cat([u, v], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _rope(s):
    c = s["case"]
    cos, sin = _cos_sin(s, c["pass"] == "bwd")
    return {n: _turn(s[n].float(), cos, sin, c["rot"], c["interleaved"]).to(s[n].dtype) for n in ("q", "k")}


def _qknorm_fwd(s):
    c = s["case"]
    cos, sin = _cos_sin(s, False)

    def one(x, gamma):
        v = x.float()
        v = v / torch.sqrt((v * v).mean(dim=-1, keepdim=True) + EPS) * gamma.float()
        return _turn(v, cos, sin, c["rot"], c["interleaved"]).to(x.dtype)

    return {n: one(s[n], s["gamma_" + n]) for n in ("q", "k")}


def _qknorm_bwd(s):
    c = s["case"]
    cos, sin = _cos_sin(s, True)

    def one(g, x, gamma):
        u, v = _turn(g.float(), cos, sin, c["rot"], c["interleaved"]), x.float()
        rstd = 1 / torch.sqrt((v * v).mean(dim=-1, keepdim=True) + EPS)
        a, xhat = u * gamma.float(), v * rstd
        grad = rstd * (a - xhat * (a * xhat).mean(dim=-1, keepdim=True))
        return grad.to(x.dtype), (u * xhat).sum(dim=(0, 1, 2), dtype=torch.float64).to(gamma.dtype)

    q, k = (one(s["g_" + n], s[n], s["gamma_" + n]) for n in ("q", "k"))
    return {"q": q[0], "k": k[0], "gamma_q": q[1], "gamma_k": k[1]}


def _philox_round(state, number):
    """One of the ten rounds on int64 lanes that hold 32-bit words; a product past 2^63 wraps, and its bits are the same."""
    c0, c1, c2, c3, k0, k1 = state
    p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
    k0n, k1n = (k0 + number * 0x9E3779B9) & 0xFFFFFFFF, (k1 + number * 0xBB67AE85) & 0xFFFFFFFF
    return (((p1 >> 32) & 0xFFFFFFFF) ^ c1 ^ k0n, p1 & 0xFFFFFFFF, ((p0 >> 32) & 0xFFFFFFFF) ^ c3 ^ k1n, p0 & 0xFFFFFFFF,
            k0, k1)


def _fields(s, total, weights):
    """16 random bits an element: those of the states, or (the counter's top bit set) those of the weights."""
    block = torch.arange((total + 7) // 8, device="cuda")
    seed, count = s["rng"][0], s["rng"][1] + s["site"]
    start = (block & 0xFFFFFFFF, (block >> 32) + (0x80000000 if weights else 0), (count & 0xFFFFFFFF).expand_as(block),
             ((count >> 32) & 0xFFFFFFFF).expand_as(block), seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    words = torch.stack(functools.reduce(_philox_round, range(10), start)[:4], dim=1)
    return torch.stack([words & 0xFFFF, words >> 16], dim=2).reshape(-1)[:total].to(torch.int32)


def _to_e4m3(x, bits):
    """e4m3 codes of magnitudes up to 448: at nearest, or with random bits below the last kept one.  Times 2^-120 the
    type's exponents are those of float32, its subnormals too, and the code is what stands above bit 20."""
    if bits is None:
        return x.to(torch.float8_e4m3fn).view(torch.uint8).int()
    return (((x * 2.0 ** -120).view(torch.int32) + ((bits << 4) | 8)) >> 20).clamp(max=0x7E)


def _adamw(s):
    c, g = s["case"], s["g"].float()
    total = g.numel()
    lr, step, scale = s["control"].unbind()
    decay = torch.repeat_interleave(s["decays"], s["lengths"], output_size=total - s["starts"][0])
    decay = torch.nn.functional.pad(decay, (s["starts"][0], 0))
    g = g * scale
    if c["states"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * (s["m_scale"] / 448)[:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * (s["v_scale"] / 448)[:, None]).view(-1).square()
    m = m + (1 - BETA1) * (g - m)
    v = BETA2 * v + (1 - BETA2) * g * g
    root = torch.sqrt(v)
    first, second = 1 - BETA1 ** step.double(), 1 - BETA2 ** step.double()
    p = s["p"].float()
    p = p - lr * decay * p - (lr / first).float() * m / (root / torch.sqrt(second).float() + ADAM_EPS)
    if c["param"] == "bf16" and c["random"]:
        s["p"].copy_(((p.view(torch.int32) + _fields(s, total, True)) & -0x10000).view(torch.float32))
    else:
        s["p"].copy_(p)
    out = {"p": s["p"]}
    if c["copies"]:
        out["copy"] = s["copy"].copy_(p)
    if c["states"] == 32:
        return out | {"m": s["m"].copy_(m), "v": s["v"].copy_(v)}
    bits = _fields(s, total, False).view(-1, BLOCK) if c["random"] else None
    swapped = ((bits & 0xFF) << 8) | (bits >> 8) if c["random"] else None
    rows_m, rows_v = m.view(-1, BLOCK), root.view(-1, BLOCK)
    top_m, top_v = rows_m.abs().amax(dim=1, keepdim=True), rows_v.amax(dim=1, keepdim=True)
    code_m = _to_e4m3(torch.where(top_m > 0, rows_m.abs() * (448 / top_m), 0.0), bits) | ((rows_m < 0).int() << 7)
    code_v = _to_e4m3(torch.where(top_v > 0, rows_v * (448 / top_v), 0.0), swapped)
    code_v = torch.where(rows_v > 0, code_v.clamp(min=1), code_v)
    s["m"].copy_(code_m.to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
    s["v"].copy_(code_v.to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
    return out | {"m": s["m"], "v": s["v"], "m_scale": s["m_scale"].copy_(top_m.view(-1)), "v_scale": s["v_scale"].copy_(top_v.view(-1))}


def _gradnorm(s):
    norm = s["g"].double().square().sum().sqrt() * s["control"][2].double()
    return {"clip": torch.stack([norm, torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)]).float()}


# ------------------------------------------------------------------------------------------ one pass
def _own_table(s, s2a):
    """The turns of each pair, which a program computes once."""
    c = s["case"]
    table = s2a.rope_table(c["rot"], base=BASE, scaling=c["scaling"], factor=FACTOR, original_length=ORIGINAL, axes=c["axes"])
    return table.cuda()


def _own_plan(s, s2a):
    """The tensors of the step, which a program lists once."""
    c = s["case"]
    g = _views(s["g"], s["sizes"], s["starts"])
    if c["op"] == "gradnorm":
        return s2a.adamw_plan(None, g, None, None)
    p, m, v = (_views(s[n], s["sizes"], s["starts"]) for n in ("p", "m", "v"))
    scales = [None, None]
    if c["states"] == 8:
        blocks = [-(-n // BLOCK) for n in s["sizes"]]
        scales = [_views(s[n], blocks, [at // BLOCK for at in s["starts"]]) for n in ("m_scale", "v_scale")]
    return s2a.adamw_plan(p, g, m, v, scales[0], scales[1], _views(s["copy"], s["sizes"], s["starts"]) if c["copies"] else None,
                          weight_decay=s["decay"])


def run(state):
    case = state["case"]
    if own:
        from paper_2503_08154_b200 import binding as s2a
        if case["op"] in ("rope", "qknorm"):
            if "table" not in state:
                state["table"] = _own_table(state, s2a)
            rest = (state["positions"], state["table"])
            if case["op"] == "rope":
                call = s2a.s2a_rope_fwd if case["pass"] == "fwd" else s2a.s2a_rope_bwd
                call(state["q"], state["k"], state["out_q"], state["out_k"], *rest, scale=state["scale"],
                     interleaved=case["interleaved"])
                return {"q": state["out_q"], "k": state["out_k"]}
            if case["pass"] == "fwd":
                s2a.s2a_qknorm_rope_fwd(state["q"], state["k"], state["gamma_q"], state["gamma_k"], state["out_q"],
                                        state["out_k"], *rest, EPS, scale=state["scale"], interleaved=case["interleaved"])
                return {"q": state["out_q"], "k": state["out_k"]}
            if "scratch" not in state:      # a workspace that a training program keeps
                state["scratch"] = torch.empty(s2a.qknorm_rope_scratch_bytes(case["batch"], case["tokens"], case["heads_q"],
                                                                             case["heads_k"], case["head_dim"]),
                                               dtype=torch.uint8, device="cuda")
            s2a.s2a_qknorm_rope_bwd(state["g_q"], state["g_k"], state["q"], state["k"], state["gamma_q"], state["gamma_k"],
                                    state["out_q"], state["out_k"], state["grad_gamma_q"], state["grad_gamma_k"],
                                    state["scratch"], *rest, EPS, scale=state["scale"], interleaved=case["interleaved"])
            return {"q": state["out_q"], "k": state["out_k"], "gamma_q": state["grad_gamma_q"],
                    "gamma_k": state["grad_gamma_k"]}
        if "plan" not in state:
            state["plan"] = _own_plan(state, s2a)
        if case["op"] == "gradnorm":
            if "scratch" not in state:
                state["scratch"] = torch.empty(s2a.grad_norm_scratch_bytes(state["plan"]), dtype=torch.uint8, device="cuda")
            s2a.s2a_grad_norm(state["plan"], state["control"], MAX_NORM, state["clip"], state["scratch"])
            return {"clip": state["clip"]}
        s2a.s2a_adamw_step(state["plan"], state["control"], BETA1, BETA2, ADAM_EPS, rng=state.get("rng"),
                           site=state.get("site", 0))
        return {n: state[n] for n in ("p", "copy", "m", "v", "m_scale", "v_scale") if n in state}
    if case["op"] == "rope":
        return _rope(state)
    if case["op"] == "qknorm":
        return _qknorm_fwd(state) if case["pass"] == "fwd" else _qknorm_bwd(state)
    return _adamw(state) if case["op"] == "adamw" else _gradnorm(state)


# ------------------------------------------------------------------------------------------ 64 bits
def _exact_phases(s, case, at, to):
    """exp(i angle) * scale of the tokens at .. to of every sequence: [batch, to - at, 1, pairs]."""
    pairs = case["rot"] // 2
    each = pairs // case["axes"]
    index = torch.arange(pairs, device="cuda", dtype=torch.float64) % each
    w = torch.exp(-math.log(BASE) * index / each)
    if case["scaling"] == "linear":
        w = w * (1 / FACTOR)
    elif case["scaling"] == "parts":
        turns = ORIGINAL * w / math.tau
        part = torch.clip((turns - 1) / 31, 0.0, 1.0)
        w = w * (part + (1 - part) / FACTOR)
    p = s["positions"] if case["axes"] == 2 else s["positions"][None]
    p = p[:, :, at:to].double().repeat_interleave(each, dim=0).permute(1, 2, 0)        # [batch, tokens, pairs]
    return torch.polar(torch.full_like(p, s["scale"]), p * w)[:, :, None]


def _exact_turn(x, phase, case):
    """The pairs as complex numbers, multiplied by their phase."""
    rot = case["rot"]
    if case["interleaved"]:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * phase
        front = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * phase
        front = torch.cat([z.real, z.imag], dim=-1)
    return torch.cat([front, x[..., rot:]], dim=-1)


def _exact_attention(s, case):
    out = {"q": [], "k": []}
    totals = {"gamma_q": 0.0, "gamma_k": 0.0}
    step = max(1, (1 << 24) // (case["batch"] * max(case["heads_q"], case["heads_k"]) * case["head_dim"]))
    for at in range(0, case["tokens"], step):
        to = min(case["tokens"], at + step)
        phase = _exact_phases(s, case, at, to)
        for n in ("q", "k"):
            x = s[n][:, at:to].double()
            if case["op"] == "rope":
                out[n].append(_exact_turn(x, phase if case["pass"] == "fwd" else phase.conj(), case))
                continue
            gamma = s["gamma_" + n].double()
            rstd = (x.square().sum(-1, keepdim=True) / case["head_dim"] + EPS) ** -0.5
            if case["pass"] == "fwd":
                out[n].append(_exact_turn(x * gamma * rstd, phase, case))
                continue
            u = _exact_turn(s["g_" + n][:, at:to].double(), phase.conj(), case)
            along = (u * gamma * x).sum(-1, keepdim=True) / case["head_dim"]
            out[n].append(u * gamma * rstd - x * along * rstd ** 3)
            totals["gamma_" + n] = totals["gamma_" + n] + (u * x * rstd).sum((0, 1, 2))
    result = {n: torch.cat(v, dim=1) for n, v in out.items()}
    return result | totals if case["op"] == "qknorm" and case["pass"] == "bwd" else result


def _philox_by_halves(counter, key):
    """Philox4x32-10 with every 32 x 32-bit product put together from 16-bit halves, so that nothing wraps."""
    low = 0xFFFFFFFF

    def product(a, m):
        ml, mh = m & 0xFFFF, m >> 16
        al, ah = a & 0xFFFF, a >> 16
        bottom, cross = al * ml, ah * ml
        middle = (bottom >> 16) + (cross & 0xFFFF) + al * mh
        return ah * mh + (cross >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) | (bottom & 0xFFFF)

    c, k = list(counter), list(key)
    for _ in range(10):
        high0, low0 = product(c[0], 0xD2511F53)
        high1, low1 = product(c[2], 0xCD9E8D57)
        c = [high1 ^ c[1] ^ k[0], low1, high0 ^ c[3] ^ k[1], low0]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def _exact_draws(s, at, count, weights):
    seed, offset = (int(v) for v in s["rng"].tolist())
    number = offset + s["site"]
    block = torch.arange(at // 8, (at + count + 7) // 8, device="cuda")
    words = _philox_by_halves([block % (1 << 32), block // (1 << 32) + ((1 << 31) if weights else 0), number % (1 << 32),
                               number >> 32], [seed % (1 << 32), seed >> 32])
    draws = torch.empty((block.numel(), 8), dtype=torch.int64, device="cuda")
    for i in range(8):
        draws[:, i] = (words[i // 2] >> (16 * (i % 2))) % 65536
    return draws.view(-1)[:count]


def _exact_e4m3(x, draws):
    """Non-negative values up to 448 on the grid of 3 bits behind the first, whose smallest step is 2^-9."""
    _, exponent = torch.frexp(x)
    unit = torch.exp2((exponent - 1).clamp(min=-6).double() - 3)
    count = x / unit
    count = torch.round(count) if draws is None else torch.floor(count + (draws + 0.5) / 65536)
    return (count * unit).clamp(max=448.0)


def _exact_adamw(s, case):
    total = s["g"].numel()
    lr, step, scale = s["control"].double().tolist()
    decay = torch.zeros(total, dtype=torch.float32, device="cuda")
    for view, value in zip(_views(decay, s["sizes"], s["starts"]), s["decay"]):
        view.fill_(value)
    names = ["p", "m", "v"] + (["copy"] if case["copies"] else []) + (["m_scale", "v_scale"] if case["states"] == 8 else [])
    out = {n: [] for n in names}
    size = 1 << 24
    for at in range(0, total, size):
        to = min(total, at + size)
        g, p = s["g"][at:to].double() * scale, s["p"][at:to].double()
        m, v = s["m"][at:to].double(), s["v"][at:to].double()
        if case["states"] == 8:
            m = m * (s["m_scale"][at // BLOCK:to // BLOCK].double() / 448).repeat_interleave(BLOCK)
            v = (v * (s["v_scale"][at // BLOCK:to // BLOCK].double() / 448).repeat_interleave(BLOCK)) ** 2
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
        p = (1 - lr * decay[at:to].double()) * p - lr * (m / (1 - BETA1 ** step)) / ((v / (1 - BETA2 ** step)).sqrt() + ADAM_EPS)
        if case["copies"]:
            out["copy"].append(p)
        if case["param"] == "bf16" and case["random"]:
            _, exponent = torch.frexp(p.abs())
            unit = torch.exp2((exponent - 8).clamp(min=-133).double())
            kept = torch.floor(p.abs() / unit + _exact_draws(s, at, to - at, True).double() / 65536) * unit
            p = torch.where(p < 0, -kept, kept)
        out["p"].append(p)
        if case["states"] == 32:
            out["m"].append(m)
            out["v"].append(v)
            continue
        bits = _exact_draws(s, at, to - at, False) if case["random"] else None
        other = (bits % 256) * 256 + bits // 256 if case["random"] else None
        for name, x, draws in (("m", m, bits), ("v", v.sqrt(), other)):
            top = x.abs().view(-1, BLOCK).max(dim=1).values
            unit = torch.where(top > 0, 448 / top, 0.0).repeat_interleave(BLOCK)
            code = _exact_e4m3(x.abs() * unit, draws)
            if name == "v":
                code = torch.where(x > 0, code.clamp(min=2.0 ** -9), code)
            out[name].append(torch.where(x < 0, -code, code))
            out[name + "_scale"].append(top)
    return {n: torch.cat(v) for n, v in out.items()}


def _exact_gradnorm(s, case):
    total = 0.0
    for at in range(0, s["g"].numel(), 1 << 25):
        total += float((s["g"][at:at + (1 << 25)].double() ** 2).sum())
    norm = math.sqrt(total) * float(s["control"][2])
    return {"clip": torch.tensor([norm, min(1.0, MAX_NORM / (norm + 1e-6))], dtype=torch.float64, device="cuda")}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rope", "qknorm"):
        return _exact_attention(s, case)
    return _exact_adamw(s, case) if case["op"] == "adamw" else _exact_gradnorm(s, case)
