"""The work of a training step beside the gradient codec, as cases that can be timed: the server's AdamW step over many tensors,
with its states in 32 or in 8 bits, and the layer norm of a model over tokens, forward and backward.

  norm    rows of a batch are normalised, scaled and shifted; their means and reciprocal deviations are kept
  grad    the gradient of the rows, and of the scale and the shift, summed over all rows
  adamw   parameters, gradients and two states in 32 bits: one step
  adamw8  the same with the states in 8 bits, a scale for each state and block of 256 elements

`own` chooses between the plain form and the framework's calls.

The states in 8 bits: m is e4m3 times a scale, v is e5m2 times a scale.  They are rounded to one of the two neighbours on their
grid at random, without bias; the random bits are Philox4x32-10's, with the seed as its key and (group, 0xFFFFFFFF, step) as
its counter.  A group is the 8 elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3 of a block, l = 0..31, and its number 32 times
the block's number in the whole list, plus l.  The element in place s of its group takes half s % 2 of word s / 2, v with its two
bytes swapped.  A v above zero is never rounded to zero.
"""
import math
import random

import torch

own = False

# Tensors of the training loop's network: three 3x3 convolutions, two fully connected layers, weights and biases.
CNN = [864, 32, 18_432, 64, 73_728, 128, 524_288, 256, 2_560, 10]
# The layered benchmark gradient: five convolutions and three fully connected layers.
ALEXNET = [34_848, 96, 307_200, 256, 884_736, 384, 663_552, 384, 442_368, 256,
           37_748_736, 4_096, 16_777_216, 4_096, 4_096_000, 1_000]
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-4, 0.1
NORM_EPS = 1e-5
BLOCK, TOP_M, TOP_V, LEAST = 256, 448.0, 57344.0, 2.0 ** -110


def listed():
    return [
        # One position of each of 64 sequences: a few rows, latency.
        {"name": "norm_64", "op": "norm", "rows": 64, "dim": 4_096, "x": "bf16", "y": "bf16", "weights": "f32"},
        # A training batch of rows looked up in bf16.
        {"name": "norm_batch_16k", "op": "norm", "rows": 16_384, "dim": 1_024, "x": "bf16", "y": "bf16", "weights": "f32"},
        # Rows of an odd length in fp32: no vector starts on a boundary.
        {"name": "norm_odd", "op": "norm", "rows": 10_007, "dim": 515, "x": "f32", "y": "f32", "weights": "f32"},
        # The training loop's model over tokens, one worker's batch: latency.
        {"name": "grad_small", "op": "grad", "rows": 2_048, "dim": 64, "x": "f32", "y": "f32", "weights": "f32", "add": False},
        # A training batch.
        {"name": "grad_batch_16k", "op": "grad", "rows": 16_384, "dim": 1_024, "x": "bf16", "y": "bf16", "weights": "f32",
         "add": False},
        # A long batch of wide rows; the weights' gradients add up over its parts.
        {"name": "grad_long_64k", "op": "grad", "rows": 65_536, "dim": 4_096, "x": "bf16", "y": "bf16", "weights": "f32",
         "add": True},
        # The server of the package's training loop, every iteration: ten small tensors.
        {"name": "adamw_cnn_620k", "op": "adamw", "tensors": "cnn", "params": "f32", "grads": "f32", "factor": 1.0},
        # The server's step at the size of the headline benchmark: the sum of 8 workers, clipped.
        {"name": "adamw_server_25M", "op": "adamw", "tensors": "split", "n": 25_000_000, "parts": 1, "params": "f32",
         "grads": "f32", "factor": 0.37},
        # A model of 61 M parameters, fp32 parameters and bf16 gradients.
        {"name": "adamw_layers_61M", "op": "adamw", "tensors": "alexnet", "params": "f32", "grads": "bf16", "factor": 1.0},
        # The training loop's server again, with states of 2 bytes a parameter.
        {"name": "adamw8_cnn_620k", "op": "adamw8", "tensors": "cnn", "params": "f32", "grads": "f32", "factor": 1.0},
        # Hundreds of tensors of odd sizes, one behind the other: most start off the boundaries.
        {"name": "adamw8_ragged_8M", "op": "adamw8", "tensors": "split", "n": 8_000_003, "parts": 301, "params": "f32",
         "grads": "f32", "factor": 0.5},
        # A model whose states would not fit in 32 bits beside the rest.
        {"name": "adamw8_100M", "op": "adamw8", "tensors": "split", "n": 100_000_000, "parts": 40, "params": "f32",
         "grads": "bf16", "factor": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "grad", "grad", "adamw", "adamw", "adamw8", "adamw8"))
    if op in ("norm", "grad"):
        dim = _log(rng, 4, 16_384)
        if rng.random() < 0.7:
            dim = (dim + 7) // 8 * 8
        case = {"op": op, "rows": min(_log(rng, 1, 131_072), 100_000_000 // dim), "dim": dim, "x": rng.choice(("f32", "bf16")),
                "y": rng.choice(("f32", "bf16")), "weights": rng.choice(("f32", "f32", "bf16"))}
        if op == "grad":
            case["add"] = rng.random() < 0.4
        return case
    n = _log(rng, 1_000, 50_000_000)
    n -= n % rng.choice((1, 8, 64))
    return {"op": op, "tensors": "split", "n": n, "parts": _log(rng, 1, min(n // 64, 600)), "params": rng.choice(("f32", "f32", "bf16")),
            "grads": rng.choice(("f32", "bf16")), "factor": rng.choice((1.0, 0.25, 0.9))}


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _sizes(case):
    """Tensor sizes in order: weight matrices of very unlike sizes, every second tensor as short as a bias vector."""
    if case["tensors"] == "cnn":
        return CNN
    if case["tensors"] == "alexnet":
        return ALEXNET
    n, parts = case["n"], case["parts"]
    weight = [((7 * i) % 13 + 1) ** 2 if i % 2 == 0 else 0.05 for i in range(parts)]
    sizes = [max(1, int(n * w / sum(weight))) for w in weight]
    if n % 8 == 0:
        sizes = [max(8, s // 8 * 8) for s in sizes]
    sizes[0] += max(0, n - sum(sizes))
    return sizes


def _slices(flat, sizes):
    at, parts = 0, []
    for s in sizes:
        parts.append(flat[at:at + s])
        at += s
    return parts


def prepare(case, seed):
    s = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, scale, kind, shift=0.0):
        return torch.empty(shape, dtype=_type(kind), device="cuda").normal_(shift, scale, generator=gen)

    if case["op"] in ("norm", "grad"):
        rows, dim = case["rows"], case["dim"]
        s["x"] = normal((rows, dim), 1.0, case["x"], 0.1)
        s["weight"], s["bias"] = normal(dim, 0.2, case["weights"], 1.0), normal(dim, 0.1, case["weights"])
        s["stats"] = torch.zeros(rows, 2, device="cuda")
        if case["op"] == "norm":
            s["out"] = torch.zeros(rows, dim, dtype=_type(case["y"]), device="cuda")
            return s
        s["dy"] = normal((rows, dim), 1e-3, case["y"])
        mean, rstd = _moments(s["x"].float())
        s["stats"].copy_(torch.cat([mean, rstd], 1))
        s["dx"] = torch.zeros(rows, dim, dtype=_type(case["x"]), device="cuda")
        s["dweight"], s["dbias"] = normal(dim, 1e-2, "f32"), normal(dim, 1e-2, "f32")
        return s
    rng = random.Random(seed)
    sizes = _sizes(case)
    n = sum(sizes)
    sigma = [10.0 ** rng.uniform(-5, -2) for _ in sizes]
    s["sizes"], s["step"], s["seed"] = sizes, rng.randrange(10, 2_000), seed
    s["decays"] = [DECAY if k % 2 == 0 else 0.0 for k in range(len(sizes))]       # every second tensor is a bias
    s["flat"] = {"params": normal(n, 0.05, case["params"]), "grads": normal(n, 1.0, case["grads"])}
    for g, sd in zip(_slices(s["flat"]["grads"], sizes), sigma):
        g.mul_(sd)
    s["factor"] = torch.tensor([case["factor"]], device="cuda")
    past = torch.randn(n, generator=gen, device="cuda")       # what the gradients were until now
    if case["op"] == "adamw":
        spread = torch.rand(n, generator=gen, device="cuda").mul_(2.0).add_(0.1)
        s["flat"]["m"], s["flat"]["v"] = past.mul_(0.3), spread
        for m, v, sd in zip(_slices(past, sizes), _slices(spread, sizes), sigma):
            m.mul_(sd)
            v.mul_(sd * sd)
    else:
        s["blocks"] = [-(-k // BLOCK) for k in sizes]
        spread = torch.rand(n, generator=gen, device="cuda").mul_(4.0).sub_(3.0).exp_()
        s["flat"]["m"] = past.mul_(TOP_M / 5.0).clamp_(-TOP_M, TOP_M).to(torch.float8_e4m3fn)
        s["flat"]["v"] = spread.mul_(TOP_V / 2.8).clamp_(0.0, TOP_V).to(torch.float8_e5m2)
        scales = torch.rand(sum(s["blocks"]), 2, generator=gen, device="cuda").add_(0.5)
        for c, sd in zip(_slices(scales, s["blocks"]), sigma):
            c.mul_(torch.tensor([1.5 * sd / TOP_M, 2.0 * sd * sd / TOP_V], device="cuda"))
        s["flat"]["scales"] = scales
    s["tensors"] = {k: _slices(v, s["blocks"] if k == "scales" else sizes) for k, v in s["flat"].items()}
    return s


def _moments(x):
    mean = x.double().mean(1, keepdim=True)
    return mean.float(), torch.rsqrt((x.double() - mean).square().mean(1, keepdim=True) + NORM_EPS).float()


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / (centred.square().mean(1, keepdim=True) + NORM_EPS).sqrt()
    y = centred * rstd * s["weight"].float() + s["bias"].float()
    return {"y": y.to(s["out"].dtype), "stats": torch.cat([mean, rstd], 1)}


def _plain_grad(s):
    dy, rstd = s["dy"].float(), s["stats"][:, 1:]
    xhat = (s["x"].float() - s["stats"][:, :1]) * rstd
    a = dy * s["weight"].float()
    dx = (a - a.mean(1, keepdim=True) - xhat * (a * xhat).mean(1, keepdim=True)) * rstd
    dweight, dbias = (dy * xhat).sum(0, dtype=torch.float64), dy.sum(0, dtype=torch.float64)
    if s["add"]:
        s["dweight"].copy_(s["dweight"].double() + dweight)
        s["dbias"].copy_(s["dbias"].double() + dbias)
    else:
        s["dweight"].copy_(dweight)
        s["dbias"].copy_(dbias)
    return {"dx": dx.to(s["x"].dtype), "dweight": s["dweight"], "dbias": s["dbias"]}


def _plain_update(s, m, v):
    """One step's m, v (32 bits) and parameters."""
    f = s["flat"]
    g = f["grads"].float() * s["factor"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * (1.0 - BETA2) * g
    c1, c2 = torch.tensor([1.0 - BETA1 ** s["step"], 1.0 - BETA2 ** s["step"]]).unbind()
    size, root = float(torch.tensor(LR) / c1), float(1.0 / c2.sqrt())
    decay = torch.tensor(s["decays"], device="cuda").mul_(LR).repeat_interleave(torch.tensor(s["sizes"], device="cuda"))
    p = f["params"].float()
    f["params"].copy_(p - (decay * p + m / (v.sqrt() * root + EPS) * size))
    return m, v


def _plain_philox(group, seed, step):
    """Four words of 32 bits for every group, in 64-bit integers."""
    low = 0xFFFFFFFF
    c = [group & low, group >> 32, torch.full_like(group, low), torch.full_like(group, step)]
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [p1 >> 32 & low ^ c[1] ^ k0, p1 & low, p0 >> 32 & low ^ c[3] ^ k1, p0 & low]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return c


def _plain_pack(x, top, h, shift):
    """Magnitudes x [blocks, 256] on the grid of a float whose last bit is bit `shift` of fp32's, times 2^-120 (e4m3) or 2^-112."""
    most = x.amax(1, keepdim=True)
    held, top = most >= LEAST, torch.full_like(most, top)           # (a division by a number would be a product)
    scale = torch.where(held, most / top, 0.0)
    y = x * torch.where(held, top / most, 0.0) * 2.0 ** (-120 if shift == 20 else -112)
    bits = y.view(torch.int32)
    return scale, bits, bits + (h << shift - 16 | 1 << shift - 17) >> shift


def _plain_adamw8(s):
    f = s["flat"]
    sizes, blocks = (torch.tensor(s[k], device="cuda") for k in ("sizes", "blocks"))
    # element i of the list lies in place at[i] of the list of whole blocks
    shift = BLOCK * (blocks.cumsum(0) - blocks) - (sizes.cumsum(0) - sizes)
    at = torch.arange(f["params"].numel(), device="cuda") + shift.repeat_interleave(sizes)
    of = at // BLOCK
    m, v = _plain_update(s, f["m"].float() * f["scales"][of, 0], f["v"].float() * f["scales"][of, 1])
    count = f["scales"].shape[0]
    group = torch.arange(count * 32, device="cuda")
    words = torch.stack(_plain_philox(group, s["seed"], s["step"])).view(4, count, 32)
    halves = torch.stack([words & 0xFFFF, words >> 16], 1).view(2, 4, count, 32)               # place s of a group: [s // 4, s % 4]
    h = halves.permute(2, 0, 3, 1).reshape(count, BLOCK).to(torch.int32)
    whole = [torch.zeros(count * BLOCK, device="cuda").index_put_((at,), w).view(count, BLOCK) for w in (m, v)]
    scale_m, _, code_m = _plain_pack(whole[0].abs(), TOP_M, h, 20)
    scale_v, bits_v, code_v = _plain_pack(whole[1], TOP_V, (h & 0xFF) << 8 | h >> 8, 21)
    code_m |= (whole[0] < 0).to(torch.int32) << 7
    code_v = torch.where((code_v == 0) & (bits_v > 0), 1, code_v)
    f["m"].view(torch.uint8).copy_(code_m.view(-1)[at])
    f["v"].view(torch.uint8).copy_(code_v.view(-1)[at])
    f["scales"].copy_(torch.cat([scale_m, scale_v], 1))


def _plain(s):
    if s["op"] == "norm":
        return _plain_norm(s)
    if s["op"] == "grad":
        return _plain_grad(s)
    if s["op"] == "adamw":
        m, v = _plain_update(s, s["flat"]["m"], s["flat"]["v"])
        s["flat"]["m"].copy_(m)
        s["flat"]["v"].copy_(v)
    else:
        _plain_adamw8(s)
    return {k: v for k, v in s["flat"].items() if k != "grads"}


def _own(s):
    import paper_1804_08066_b200 as mqg
    if s["op"] == "norm":
        mqg.mqg_layer_norm(s["x"], s["rows"], s["dim"], s["weight"], s["bias"], NORM_EPS, s["out"], s["stats"])
        return {"y": s["out"], "stats": s["stats"]}
    if s["op"] == "grad":
        if "workspace" not in s:             # scratch memory, which a program keeps from step to step
            s["workspace"] = torch.empty(max(1, mqg.mqg_layer_norm_workspace_floats(s["rows"], s["dim"])), device="cuda")
        mqg.mqg_layer_norm_grad(s["dy"], s["x"], s["rows"], s["dim"], s["weight"], s["stats"], s["dx"], s["dweight"], s["dbias"],
                                s["workspace"], add_into_grads=s["add"])
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    t = s["tensors"]
    if s["op"] == "adamw":
        mqg.mqg_adamw(t["params"], t["grads"], t["m"], t["v"], s["decays"], LR, BETA1, BETA2, EPS, s["step"], factor=s["factor"])
    else:
        mqg.mqg_adamw8(t["params"], t["grads"], t["m"], t["v"], t["scales"], s["decays"], LR, BETA1, BETA2, EPS, s["step"],
                       s["seed"], factor=s["factor"])
    return {k: v for k, v in s["flat"].items() if k != "grads"}


def run(state):
    out = _own(state) if own else _plain(state)
    if "step" in state:
        state["step"] += 1
    return out


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] in ("norm", "grad"):
        rows, dim, weights = case["rows"], case["dim"], case["dim"] * size[case["weights"]]
        n = rows * dim
        if case["op"] == "norm":
            return {"bytes": n * (size[case["x"]] + size[case["y"]]) + 2 * weights + 8 * rows, "flops": 7 * n}
        return {"bytes": n * (2 * size[case["x"]] + size[case["y"]]) + weights + 8 * rows + (16 if case["add"] else 8) * dim,
                "flops": 13 * n}
    sizes = _sizes(case)
    n = sum(sizes)
    states = 16 * n if case["op"] == "adamw" else 4 * n + 16 * sum(-(-k // BLOCK) for k in sizes)
    return {"bytes": n * (2 * size[case["params"]] + size[case["grads"]]) + states, "flops": (15 if case["op"] == "adamw" else 30) * n}


def _exact_words(group, seed, step):
    """Philox4x32-10 by products of 16-bit halves, which no integer of 64 bits overflows."""
    def product(a, b):
        low, high = (a & 0xFFFF) * b, (a >> 16) * b
        total_high, carry = high >> 16, ((high & 0xFFFF) << 16) + low
        return total_high + (carry >> 32), carry & 0xFFFFFFFF

    x0, x1, x2, x3 = group % 2 ** 32, group // 2 ** 32, group * 0 + (2 ** 32 - 1), group * 0 + step
    for r in range(10):
        key = (seed + r * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        (h0, l0), (h1, l1) = product(x0, 0xD2511F53), product(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ key[0], l1, h0 ^ x3 ^ key[1], l0
    return x0, x1, x2, x3


def _exact_rounded(y, u, fraction, least):
    """y >= 0 on the grid of a float with `fraction` bits behind the point and 2^least as its smallest normal number: rounded up
    where u, even in (0, 1), is at least one minus what is above the lower neighbour."""
    exponent = torch.frexp(y)[1] - 1
    step = torch.ldexp(torch.ones_like(y), exponent.clamp(min=least) - fraction)
    return torch.floor(y / step + u) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, dim = s["x"].double(), case["dim"]
        mean = x.sum(1) / dim
        x -= mean[:, None]
        rstd = ((x * x).sum(1) / dim + NORM_EPS) ** -0.5
        y = torch.addcmul(s["bias"].double(), x.mul_(rstd[:, None]), s["weight"].double())
        return {"y": y, "stats": torch.stack([mean, rstd], 1)}
    if case["op"] == "grad":
        x, dy, dim = s["x"].double(), s["dy"].double(), case["dim"]
        mean, rstd = (c.double()[:, None] for c in s["stats"].unbind(1))
        x.sub_(mean).mul_(rstd)
        kept = 1.0 if case["add"] else 0.0
        out = {"dweight": kept * s["dweight"].double() + (dy * x).sum(0), "dbias": kept * s["dbias"].double() + dy.sum(0)}
        dy *= s["weight"].double()
        along, around = (dy * x).sum(1, keepdim=True) / dim, dy.sum(1, keepdim=True) / dim
        out["dx"] = dy.sub_(around).sub_(x.mul_(along)).mul_(rstd)
        return out
    f, t = s["flat"], s["step"]
    sizes = torch.tensor(s["sizes"])
    tensor = torch.repeat_interleave(torch.arange(len(s["sizes"])), sizes).cuda()
    p, g = f["params"].double(), f["grads"].double() * s["factor"].double()
    m, v = f["m"].double(), f["v"].double()
    if case["op"] == "adamw8":
        place = torch.arange(p.numel(), device="cuda") - (sizes.cumsum(0) - sizes).cuda()[tensor]       # in its tensor
        first = torch.tensor(s["blocks"]).cumsum(0) - torch.tensor(s["blocks"])
        block = first.cuda()[tensor] + place // BLOCK
        m *= f["scales"].double()[block, 0]
        v *= f["scales"].double()[block, 1]
    m = m.mul_(BETA1).add_(g, alpha=1.0 - BETA1)
    v = v.mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
    rate = torch.tensor(s["decays"], dtype=torch.float64, device="cuda")[tensor] * LR
    p -= rate * p + LR / (1.0 - BETA1 ** t) * m / ((v / (1.0 - BETA2 ** t)).sqrt() + EPS)
    out = {"params": p, "m": m, "v": v}
    if case["op"] == "adamw":
        return out
    within = place % BLOCK
    group = block * 32 + within % 128 // 4
    slot = within // 128 * 4 + within % 4
    words = torch.stack(_exact_words(torch.arange(f["scales"].shape[0] * 32, device="cuda"), seed, t))
    h = words[slot // 2, group] >> 16 * (slot % 2) & 0xFFFF
    scales = torch.zeros(f["scales"].shape, dtype=torch.float64, device="cuda")
    for k, (x, top, draws, fraction, least) in enumerate(((m.abs(), TOP_M, h, 3, -6),
                                                         (v, TOP_V, h % 256 * 256 + h // 256, 2, -14))):
        most = scales[:, k].scatter_reduce(0, block, x, "amax")
        scales[:, k] = torch.where(most >= LEAST, most / top, 0.0)
        unit = torch.where(most >= LEAST, top / most, 0.0)[block]
        q = _exact_rounded(x * unit, (draws.double() + 0.5) / 65536.0, fraction, least)
        out["mv"[k]] = torch.copysign(q, m) if k == 0 else torch.where((q == 0) & (x * unit > 0), 2.0 ** (least - fraction), q)
    out["scales"] = scales
    return out
