"""The layers that sit between the stash kernels in a transformer block: layer norm, dropout and the
bucketed relative position bias, each with its backward pass.

Every operator has its plain form here (elementary torch operations in 32 bits, 64 where a sum is long or an
index is hashed) beside the call that a user makes of this repository's kernels (``own`` is true).

* layer norm: mean and 1/sqrt(var + eps) of each row; y = (x - mean) * rstd * gamma + beta.  Backward, from x and the
  (mean, rstd) that the forward pass kept: a = g * gamma, xhat = (x - mean) * rstd,
  grad_x = rstd * (a - mean(a) - xhat * mean(a * xhat)), grad_gamma = sum over rows of g * xhat,
  grad_beta = sum over rows of g.
* dropout: element e takes 16 bits of Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3",
  2011) at counter (e / 8, offset + site) under the key `seed`; it is kept when they are at least
  T = round(65536 p), and then scaled by 65536 / (65536 - T).  Nothing is stored: backward draws the same bits again.
* relative position bias: y[b, h, q, k] = x[b, h, q, k] + table[bucket(q, k), h], bucket given as a [tq, tk] map (2-D
  windows) or as a vector over the distance k - q (1-D sequences); grad_table[u, h] is the sum of grad_out over the
  batch and over the positions of bucket u.
"""
import functools
import math

import torch

own = False

EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the class tokens' final norm of a batch: one strided row per image; latency is all that counts
        {"name": "norm_fwd_class_tokens", "op": "norm", "pass": "fwd", "dtype": "f32", "weights": "f32", "rows": 64,
         "row_len": 768, "stride": 197 * 768, "frozen": False},
        # a ViT-B/16 block's norm, batch 64, bfloat16 activations under float32 weights
        {"name": "norm_fwd_vit_b", "op": "norm", "pass": "fwd", "dtype": "bf16", "weights": "f32", "rows": 64 * 197,
         "row_len": 768, "stride": 768, "frozen": False},
        # the same norm's backward pass with both weights' gradients
        {"name": "norm_bwd_vit_b", "op": "norm", "pass": "bwd", "dtype": "bf16", "weights": "f32", "rows": 64 * 197,
         "row_len": 768, "stride": 768, "frozen": False},
        # an odd row length in float32, where no row but every fourth starts on a 16-byte boundary
        {"name": "norm_bwd_odd_f32", "op": "norm", "pass": "bwd", "dtype": "f32", "weights": "f32", "rows": 8 * 577,
         "row_len": 1025, "stride": 1025, "frozen": False},
        # a long sequence at a wide model width, everything in bfloat16: the largest norm
        {"name": "norm_bwd_wide", "op": "norm", "pass": "bwd", "dtype": "bf16", "weights": "bf16", "rows": 64 * 1024,
         "row_len": 4096, "stride": 4096, "frozen": False},
        # one image's residual branch
        {"name": "dropout_residual_one_image", "op": "dropout", "pass": "fwd", "dtype": "f32", "n": 197 * 768,
         "residual": True, "p": 0.1},
        # attention probabilities of a ViT-B/16 block, batch 64
        {"name": "dropout_fwd_attention_vit_b", "op": "dropout", "pass": "fwd", "dtype": "bf16", "n": 64 * 12 * 197 * 197,
         "residual": False, "p": 0.1},
        # the gradient of a long activation whose length ends inside a vector
        {"name": "dropout_bwd_long_odd", "op": "dropout", "pass": "bwd", "dtype": "bf16", "n": 200_000_003,
         "residual": False, "p": 0.5},
        # attention scores of a ViT-B/16 block with the 2-D window's 732 buckets (14 x 14 patches and a class token)
        {"name": "bias_fwd_window_vit_b", "op": "bias", "pass": "fwd", "dtype": "bf16", "weights": "f32", "batch": 64,
         "heads": 12, "tq": 197, "tk": 197, "form": "window", "buckets": 732},
        # and the gradient of its table
        {"name": "bias_bwd_window_vit_b", "op": "bias", "pass": "bwd", "dtype": "bf16", "weights": "f32", "batch": 64,
         "heads": 12, "tq": 197, "tk": 197, "form": "window", "buckets": 732},
        # the table's gradient over a long sequence: little batch to sum over first, buckets of millions of positions
        {"name": "bias_bwd_long", "op": "bias", "pass": "bwd", "dtype": "bf16", "weights": "bf16", "batch": 2,
         "heads": 16, "tq": 2048, "tk": 2048, "form": "distance", "buckets": 32},
        # one new token per sequence against a cache of 4097 keys
        {"name": "bias_fwd_one_token", "op": "bias", "pass": "fwd", "dtype": "bf16", "weights": "f32", "batch": 64,
         "heads": 16, "tq": 1, "tk": 4097, "form": "distance", "buckets": 32},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["norm", "dropout", "bias"])
    case = {"op": op, "pass": rng.choice(["fwd", "bwd"]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "norm":
        row_len = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            row_len = max(16, row_len // 16 * 16)
        rows = _log_int(rng, 1, max(1, (1 << 26) // row_len))
        case |= {"weights": rng.choice(["bf16", "f32"]), "rows": rows, "row_len": row_len,
                 "stride": row_len + rng.choice([0, 0, 0, 8, 24]), "frozen": rng.random() < 0.25}
    elif op == "dropout":
        case |= {"n": _log_int(rng, 1, 150_000_000), "residual": case["pass"] == "fwd" and rng.random() < 0.5,
                 "p": rng.choice([0.0, 0.05, 0.1, 0.3, 0.5, 0.9])}
    else:
        case |= {"weights": rng.choice(["bf16", "f32"]), "heads": rng.choice([1, 3, 6, 12, 16])}
        if rng.random() < 0.5:
            side = rng.randint(2, 20)
            t = side * side + 1
            case |= {"tq": t, "tk": t, "form": "window", "buckets": (2 * side - 1) ** 2 + 3}
        else:
            tk = _log_int(rng, 1, 2048)
            case |= {"tq": rng.choice([1, tk, max(1, tk // 3)]), "tk": tk, "form": "distance",
                     "buckets": rng.choice([8, 32, 64])}
        case["batch"] = _log_int(rng, 1, max(1, min(128, (1 << 26) // (case["heads"] * case["tq"] * case["tk"]))))
    return case


def work(case):
    s = SIZE[case["dtype"]]
    if case["op"] == "norm":
        n, w = case["rows"] * case["row_len"], SIZE[case["weights"]] * case["row_len"]
        if case["pass"] == "fwd":
            return {"bytes": 2 * n * s + 8 * case["rows"] + 2 * w, "flops": 8 * n}
        return {"bytes": 3 * n * s + 8 * case["rows"] + (w if case["frozen"] else 3 * w),
                "flops": (9 if case["frozen"] else 12) * n}
    if case["op"] == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * case["n"] * s, "flops": (2 if case["residual"] else 1) * case["n"]}
    positions = case["tq"] * case["tk"]
    n = case["batch"] * case["heads"] * positions
    small = 4 * (positions if case["form"] == "window" else case["tq"] + case["tk"] - 1)
    small += SIZE[case["weights"]] * case["buckets"] * case["heads"]
    return {"bytes": (2 if case["pass"] == "fwd" else 1) * n * s + small, "flops": n}


# ------------------------------------------------------------------------------------------ inputs
def _window_buckets(side):
    """Buckets of a side x side window behind a class token: one per (row, column) offset, and three for class-to-patch,
    patch-to-class and class-to-class."""
    at = torch.arange(side * side)
    row, col = at // side, at % side
    span = 2 * side - 1
    inner = (row[:, None] - row[None, :] + side - 1) * span + (col[:, None] - col[None, :] + side - 1)
    full = torch.full((side * side + 1, side * side + 1), span * span, dtype=torch.int64)
    full[1:, 0] = span * span + 1
    full[0, 0] = span * span + 2
    full[1:, 1:] = inner
    return full.to(torch.int32)


def _distance_buckets(tq, tk, buckets):
    """Buckets over the distance k - q, q being the last tq of tk positions: half of them for keys ahead of the query; in
    each half one bucket per short distance, then ever wider ones."""
    far = torch.arange(tq + tk - 1) - (tq - 1) - (tk - tq if tk > tq else 0)
    half = buckets // 2
    near = half // 2
    n = far.abs()
    wide = near + (torch.log2(n.clamp(min=1).double() / near) / 4 * (half - near)).long().clamp(max=half - near - 1)
    return (torch.where(n < near, n, wide) + half * (far > 0)).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0, scale, generator=gen).to(dtype)

    state = {"case": case}
    if case["op"] == "norm":
        rows, row_len = case["rows"], case["row_len"]
        spread = 0.5 + torch.rand(row_len, device="cuda", generator=gen)        # channels of unequal scale and offset
        offset = normal(row_len, scale=0.5, dtype=torch.float32)
        whole = torch.empty((rows, case["stride"]), dtype=dt, device="cuda")
        x = whole[:, :row_len]
        x.copy_(normal(rows, row_len, dtype=torch.float32).mul_(spread).add_(offset))
        wt = DTYPES[case["weights"]]
        state |= {"x": x, "gamma": (1 + normal(row_len, scale=0.2, dtype=torch.float32)).to(wt),
                  "beta": normal(row_len, scale=0.2, dtype=wt), "y": torch.empty((rows, row_len), dtype=dt, device="cuda")}
        if case["pass"] == "fwd":
            state["stats"] = torch.empty((rows, 2), dtype=torch.float32, device="cuda")
        else:
            var, mean = torch.var_mean(x.float(), dim=1, correction=0)
            state |= {"stats": torch.stack([mean, torch.rsqrt(var + EPS)], dim=1), "g": normal(rows, row_len, scale=0.01)}
            if not case["frozen"]:
                state |= {"grad_gamma": torch.empty_like(state["gamma"]), "grad_beta": torch.empty_like(state["beta"])}
    elif case["op"] == "dropout":
        n = case["n"]
        state |= {"x": normal(n), "y": torch.empty(n, dtype=dt, device="cuda"),
                  "residual": normal(n) if case["residual"] else None,
                  "rng": torch.tensor([(seed * 0x9E3779B97F4A7C15 + 0x1234567) % (1 << 63), 1000 + seed % 977],
                                      dtype=torch.int64, device="cuda"),
                  "site": 3 + seed % 11}
    else:
        b, h, tq, tk = case["batch"], case["heads"], case["tq"], case["tk"]
        wt = DTYPES[case["weights"]]
        if case["form"] == "window":
            buckets = _window_buckets(math.isqrt(tq))
        else:
            buckets = _distance_buckets(tq, tk, case["buckets"])
        state |= {"buckets": buckets.cuda(), "table": normal(case["buckets"], h, scale=0.5, dtype=wt)}
        if case["pass"] == "fwd":
            state |= {"x": normal(b, h, tq, tk, scale=2.0), "y": torch.empty((b, h, tq, tk), dtype=dt, device="cuda")}
        else:
            state |= {"g": normal(b, h, tq, tk, scale=0.01), "grad_table": torch.empty_like(state["table"])}
    return state


# ------------------------------------------------------------------------------------------ plain forms
def _norm_fwd(s):
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    centred = x - mean
    rstd = 1 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    y = centred * rstd * s["gamma"].float() + s["beta"].float()
    return {"y": y.to(s["x"].dtype), "stats": torch.cat([mean, rstd], dim=1)}


def _norm_bwd(s):
    g, mean, rstd = s["g"].float(), s["stats"][:, :1], s["stats"][:, 1:]
    xhat = (s["x"].float() - mean) * rstd
    a = g * s["gamma"].float()
    grad = rstd * (a - a.mean(dim=1, keepdim=True) - xhat * (a * xhat).mean(dim=1, keepdim=True))
    out = {"grad_x": grad.to(s["g"].dtype)}
    if not s["case"]["frozen"]:
        out["grad_gamma"] = (g * xhat).sum(dim=0).to(s["gamma"].dtype)
        out["grad_beta"] = g.sum(dim=0).to(s["gamma"].dtype)
    return out


def _philox_round(state, number):
    """One of the ten rounds on int64 lanes that hold 32-bit words; a product past 2^63 wraps, and its bits are the same."""
    c0, c1, c2, c3, k0, k1 = state
    p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
    k0n, k1n = (k0 + number * 0x9E3779B9) & 0xFFFFFFFF, (k1 + number * 0xBB67AE85) & 0xFFFFFFFF
    return (((p1 >> 32) & 0xFFFFFFFF) ^ c1 ^ k0n, p1 & 0xFFFFFFFF, ((p0 >> 32) & 0xFFFFFFFF) ^ c3 ^ k1n, p0 & 0xFFFFFFFF,
            k0, k1)


def _kept(s):
    n = s["case"]["n"]
    block = torch.arange((n + 7) // 8, device="cuda")
    seed, count = s["rng"][0], s["rng"][1] + s["site"]
    start = (block & 0xFFFFFFFF, block >> 32, (count & 0xFFFFFFFF).expand_as(block),
             ((count >> 32) & 0xFFFFFFFF).expand_as(block), seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    words = torch.stack(functools.reduce(_philox_round, range(10), start)[:4], dim=1)
    bits = torch.stack([words & 0xFFFF, words >> 16], dim=2).reshape(-1)[:n]
    return bits >= round(65536 * s["case"]["p"])


def _dropout(s):
    scale = 65536 / (65536 - round(65536 * s["case"]["p"]))
    y = torch.where(_kept(s), s["x"].float() * scale, torch.zeros((), device="cuda"))
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return {"y": y.to(s["x"].dtype)}


def _bucket_map(s):
    c = s["case"]
    if c["form"] == "window":
        return s["buckets"].long()
    at = torch.arange(c["tk"], device="cuda")[None, :] - torch.arange(c["tq"], device="cuda")[:, None] + c["tq"] - 1
    return s["buckets"].long()[at]


def _bias_fwd(s):
    bias = s["table"].float()[_bucket_map(s)].permute(2, 0, 1)
    return {"y": (s["x"].float() + bias).to(s["x"].dtype)}


def _bias_bwd(s):
    heads = s["case"]["heads"]
    summed = s["g"].sum(dim=0, dtype=torch.float64).reshape(heads, -1).t()
    table = torch.zeros(s["table"].shape, dtype=torch.float64, device="cuda")
    return {"grad_table": table.index_add_(0, _bucket_map(s).reshape(-1), summed).to(s["table"].dtype)}


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2503_08154_b200 import binding as s2a
        if case["op"] == "norm":
            if case["pass"] == "fwd":
                s2a.s2a_layernorm_fwd(state["x"], state["gamma"], state["beta"], state["y"], state["stats"],
                                      case["row_len"], EPS)
                return {"y": state["y"], "stats": state["stats"]}
            if case["frozen"]:
                s2a.s2a_layernorm_bwd(state["g"], state["x"], state["gamma"], state["stats"], state["y"], None, None, None,
                                      case["row_len"])
                return {"grad_x": state["y"]}
            if "scratch" not in state:      # a workspace that a training program keeps
                state["scratch"] = torch.empty(s2a.layernorm_scratch_bytes(case["rows"], case["row_len"]),
                                               dtype=torch.uint8, device="cuda")
            s2a.s2a_layernorm_bwd(state["g"], state["x"], state["gamma"], state["stats"], state["y"], state["grad_gamma"],
                                  state["grad_beta"], state["scratch"], case["row_len"])
            return {"grad_x": state["y"], "grad_gamma": state["grad_gamma"], "grad_beta": state["grad_beta"]}
        if case["op"] == "dropout":
            if case["pass"] == "fwd":
                s2a.s2a_dropout_fwd(state["x"], state["residual"], state["y"], state["rng"], state["site"], case["p"])
            else:
                s2a.s2a_dropout_bwd(state["x"], state["y"], state["rng"], state["site"], case["p"])
            return {"y": state["y"]}
        if case["pass"] == "fwd":
            s2a.s2a_relbias_fwd(state["x"], state["table"], state["buckets"], state["y"], case["batch"], case["heads"],
                                case["tq"], case["tk"])
            return {"y": state["y"]}
        if "scratch" not in state:
            state["scratch"] = torch.empty(s2a.relbias_scratch_bytes(case["batch"], case["heads"], case["tq"], case["tk"],
                                                                     case["buckets"]), dtype=torch.uint8, device="cuda")
        s2a.s2a_relbias_bwd(state["g"], state["buckets"], state["grad_table"], state["scratch"], case["batch"],
                            case["heads"], case["tq"], case["tk"])
        return {"grad_table": state["grad_table"]}
    if case["op"] == "norm":
        return _norm_fwd(state) if case["pass"] == "fwd" else _norm_bwd(state)
    if case["op"] == "dropout":
        return _dropout(state)
    return _bias_fwd(state) if case["pass"] == "fwd" else _bias_bwd(state)


# ------------------------------------------------------------------------------------------ 64 bits
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


def _exact_norm(s, case):
    out = {"y": [], "stats": [], "grad_x": []}
    width = case["row_len"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    total_gamma, total_beta = torch.zeros_like(gamma), torch.zeros_like(beta)
    step = max(1, (1 << 25) // width)
    for at in range(0, case["rows"], step):
        x = s["x"][at:at + step].double()
        if case["pass"] == "fwd":
            mean = x.sum(1) / width
            rstd = (((x - mean[:, None]) ** 2).sum(1) / width + EPS) ** -0.5
            out["y"].append((x - mean[:, None]) * rstd[:, None] * gamma + beta)
            out["stats"].append(torch.stack([mean, rstd], 1))
            continue
        g, kept = s["g"][at:at + step].double(), s["stats"][at:at + step].double()
        unit = (x - kept[:, :1]) * kept[:, 1:]
        weighted = g * gamma
        along = (weighted * unit).sum(1, keepdim=True) / width
        out["grad_x"].append((weighted - weighted.sum(1, keepdim=True) / width - unit * along) * kept[:, 1:])
        total_gamma += (g * unit).sum(0)
        total_beta += g.sum(0)
    result = {k: torch.cat(v) for k, v in out.items() if v}
    if case["pass"] == "bwd" and not case["frozen"]:
        result |= {"grad_gamma": total_gamma, "grad_beta": total_beta}
    return result


def _exact_dropout(s, case):
    n, threshold = case["n"], round(65536 * case["p"])
    seed, offset = (int(v) for v in s["rng"].tolist())
    count = offset + s["site"]
    y = torch.empty(n, dtype=torch.float64, device="cuda")
    step = 1 << 24                                                  # elements at a time, a multiple of eight
    for at in range(0, n, step):
        m = min(step, n - at)
        block = torch.arange(at // 8, (at + m + 7) // 8, device="cuda")
        words = _philox_by_halves([block % (1 << 32), block // (1 << 32), count % (1 << 32), count >> 32],
                                  [seed % (1 << 32), seed >> 32])
        draws = torch.empty((block.numel(), 8), dtype=torch.int64, device="cuda")
        for i in range(8):
            draws[:, i] = (words[i // 2] >> (16 * (i % 2))) % 65536
        part = s["x"][at:at + m].double() * (65536 / (65536 - threshold)) * (draws.view(-1)[:m] >= threshold)
        y[at:at + m] = part if s["residual"] is None else part + s["residual"][at:at + m].double()
    return {"y": y}


def _exact_bias(s, case):
    tq, tk = case["tq"], case["tk"]
    if case["form"] == "window":
        where = s["buckets"].long()
    else:
        rows = [s["buckets"][tq - 1 - q:tq - 1 - q + tk] for q in range(tq)]
        where = torch.stack(rows).long()
    if case["pass"] == "fwd":
        y = s["x"].double()
        for h in range(case["heads"]):
            y[:, h] += s["table"][:, h].double()[where]
        return {"y": y}
    grad = torch.empty(s["table"].shape, dtype=torch.float64, device="cuda")
    for h in range(case["heads"]):
        grad[:, h] = torch.bincount(where.reshape(-1), weights=s["g"][:, h].double().sum(0).reshape(-1),
                                    minlength=case["buckets"])
    return {"grad_table": grad}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "dropout": _exact_dropout, "bias": _exact_bias}[case["op"]](s, case)
