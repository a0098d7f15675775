"""The work of a training step around the gradient codec, as cases that can be timed: clipping by the global norm of many
gradient tensors, and the table of a model over tokens (rows looked up, and their gradient).

  flatten   a worker's gradient tensors are clipped by their common norm and written one after another into the flat
            vector that the codec encodes
  inplace   the same without the flat vector: the tensors themselves are scaled
  server    the server measures the summed gradient and applies it, clipped, to the shared parameters
  lookup    rows of the table for a batch of token ids, times a scale
  grad      the gradient of the table: rows of the output's gradient summed by token id

`own` chooses between the plain form and the framework's calls.
"""
import math
import random

import numpy as np
import torch

own = False

# Tensors of the training loop's network: three 3x3 convolutions, two fully connected layers, weights and biases.
CNN = [864, 32, 18_432, 64, 73_728, 128, 524_288, 256, 2_560, 10]
# The layered benchmark gradient: five convolutions and three fully connected layers.
ALEXNET = [34_848, 96, 307_200, 256, 884_736, 384, 663_552, 384, 442_368, 256,
           37_748_736, 4_096, 16_777_216, 4_096, 4_096_000, 1_000]


def listed():
    return [
        # A worker of the package's training loop, every iteration: ten small tensors, over the limit.
        {"name": "flatten_cnn_620k", "op": "flatten", "tensors": "cnn", "types": "f32", "out": "f32", "limit": 0.25},
        # A worker with a model of 61 M parameters in bf16, encoded as one fp32 vector.
        {"name": "flatten_layers_61M", "op": "flatten", "tensors": "alexnet", "types": "bf16", "out": "f32", "limit": 0.5},
        # Hundreds of tensors of odd sizes and both types, off the 16-byte boundaries, into a bf16 vector.
        {"name": "flatten_ragged_8M", "op": "flatten", "tensors": "split", "n": 8_000_003, "parts": 301, "types": "mixed",
         "out": "bf16", "limit": 0.1},
        # Most steps of a run that goes well: a large bf16 gradient whose norm stays within the limit.
        {"name": "inplace_within_250M", "op": "inplace", "tensors": "split", "n": 250_000_000, "parts": 40, "types": "bf16",
         "limit": 4.0},
        # The server's step for a small model: latency.
        {"name": "server_100k", "op": "server", "tensors": "split", "n": 100_013, "parts": 1, "types": "f32", "limit": 0.5},
        # The server's step at the size of the headline benchmark.
        {"name": "server_25M", "op": "server", "tensors": "split", "n": 25_000_000, "parts": 1, "types": "f32", "limit": 0.5},
        # One position of each of 64 sequences: a few rows, latency.
        {"name": "lookup_64", "op": "lookup", "rows": 32_000, "dim": 4_096, "tokens": 64, "types": "bf16", "out": "bf16",
         "ids": "i64", "spread": "zipf", "empty": 0.0},
        # A training batch from an fp32 table (the shared parameters) into bf16 activations, some places of it empty.
        {"name": "lookup_batch_16k", "op": "lookup", "rows": 50_000, "dim": 1_024, "tokens": 16_384, "types": "f32",
         "out": "bf16", "ids": "i64", "spread": "zipf", "empty": 0.05},
        # The training loop's model over tokens: a small table, one worker's batch.
        {"name": "grad_small", "op": "grad", "rows": 1_000, "dim": 64, "tokens": 2_048, "types": "f32", "out": "f32",
         "ids": "i64", "spread": "uniform", "empty": 0.1, "add": False},
        # A training batch: bf16 gradients of the activations into the table's slice of the flat fp32 gradient.
        {"name": "grad_batch_16k", "op": "grad", "rows": 50_000, "dim": 1_024, "tokens": 16_384, "types": "bf16", "out": "f32",
         "ids": "i64", "spread": "zipf", "empty": 0.05, "add": False},
        # A table shared with the output layer, whose gradient is there already; wide rows, a long batch.
        {"name": "grad_shared_64k", "op": "grad", "rows": 64_000, "dim": 4_096, "tokens": 65_536, "types": "bf16", "out": "f32",
         "ids": "i64", "spread": "zipf", "empty": 0.0, "add": True},
        # Rows of an odd length in bf16: no vector starts on a boundary.
        {"name": "grad_odd", "op": "grad", "rows": 30_011, "dim": 515, "tokens": 10_007, "types": "bf16", "out": "bf16",
         "ids": "i32", "spread": "zipf", "empty": 0.02, "add": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("flatten", "flatten", "inplace", "server", "lookup", "grad", "grad"))
    if op in ("flatten", "inplace", "server"):
        n = _log(rng, 1_000, 100_000_000)
        n -= n % rng.choice((1, 8, 64))
        parts = 1 if op == "server" else _log(rng, 1, min(n // 64, 60 if op == "inplace" else 600))
        case = {"op": op, "tensors": "split", "n": n, "parts": parts,
                "types": "f32" if op == "server" else rng.choice(("f32", "bf16", "mixed")),
                "limit": rng.choice((0.03, 0.5, 2.0))}
        if op == "flatten":
            case["out"] = rng.choice(("f32", "f32", "bf16"))
        return case
    rows, dim = _log(rng, 16, 200_000), _log(rng, 4, 8_192)
    if rng.random() < 0.7:
        dim = (dim + 7) // 8 * 8
    rows = min(rows, 200_000_000 // dim)
    tokens = min(_log(rng, 1, 131_072), 200_000_000 // dim)
    case = {"op": op, "rows": rows, "dim": dim, "tokens": tokens, "types": rng.choice(("f32", "bf16")),
            "out": rng.choice(("f32", "bf16")), "ids": rng.choice(("i64", "i32")),
            "spread": rng.choice(("zipf", "uniform")), "empty": rng.choice((0.0, 0.05, 0.5))}
    if op == "grad":
        case["add"] = rng.random() < 0.4
    return case


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


def _kinds(case, parts):
    kind = case["types"]
    return [("f32", "bf16")[i % 3 == 1] if kind == "mixed" else kind for i in range(parts)]


def _gradients(sizes, kinds, seed):
    """Slices of one vector per type, tensor j drawn from N(0, sigma_j); the vectors; sqrt(sum of size_j sigma_j^2)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    sigma = [10.0 ** rng.uniform(-5, -2) for _ in sizes]
    at = {k: 0 for k in kinds}
    store = {k: torch.empty(sum(s for s, q in zip(sizes, kinds) if q == k), dtype=_type(k), device="cuda") for k in at}
    grads = []
    for s, k, sd in zip(sizes, kinds, sigma):
        g = store[k][at[k]:at[k] + s]
        at[k] += s
        grads.append(g.normal_(0.0, sd, generator=gen))
    return grads, list(store.values()), math.sqrt(sum(s * sd * sd for s, sd in zip(sizes, sigma)))


def _token_ids(case, gen):
    """Ids as text has them (the k-th most frequent in proportion to 1 / k) or even; -1 in the empty places."""
    rows, tokens = case["rows"], case["tokens"]
    u = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
    ids = (rows ** u).floor() - 1 if case["spread"] == "zipf" else (rows * u).floor()
    ids = ids.clamp_(0, rows - 1).to(torch.int64)
    ids = torch.where(torch.rand(tokens, generator=gen, device="cuda") < case["empty"], -1, ids)
    return ids if case["ids"] == "i64" else ids.to(torch.int32)


def prepare(case, seed):
    s = dict(case)
    if case["op"] in ("flatten", "inplace", "server"):
        sizes = _sizes(case)
        s["grads"], s["vectors"], norm = _gradients(sizes, _kinds(case, len(sizes)), seed)
        s["max_norm"] = case["limit"] * norm
        s["result"] = torch.zeros(2, device="cuda")
        if case["op"] == "flatten":
            s["flat"] = torch.zeros(sum(sizes), dtype=_type(case["out"]), device="cuda")
        if case["op"] == "server":
            gen = torch.Generator(device="cuda").manual_seed(seed + 1)
            s["params"] = torch.randn(sum(sizes), generator=gen, device="cuda").mul_(0.05)
            s["lr"] = 0.1
        return s
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s["ids"] = _token_ids(case, gen)
    s["scale"] = math.sqrt(case["dim"])
    table, batch = (case["rows"], case["dim"]), (case["tokens"], case["dim"])
    if case["op"] == "lookup":
        s["table"] = torch.empty(table, dtype=_type(case["types"]), device="cuda").normal_(0.0, 0.02, generator=gen)
        s["y"] = torch.zeros(batch, dtype=_type(case["out"]), device="cuda")
    else:
        s["dout"] = torch.empty(batch, dtype=_type(case["types"]), device="cuda").normal_(0.0, 1e-3, generator=gen)
        s["grad"] = torch.empty(table, dtype=_type(case["out"]), device="cuda").normal_(0.0, 1e-3, generator=gen)
    return s


def _plain_factor(values, max_norm):
    """The norm of `values` and what it is clipped with."""
    norm = values.square().sum().sqrt()
    return norm, torch.where(norm <= max_norm, torch.ones_like(norm), max_norm / norm)


def _plain(s):
    if s["op"] == "flatten":
        x = torch.cat(s["grads"]).float()
        norm, c = _plain_factor(x, s["max_norm"])
        return {"flat": (x * c).to(s["flat"].dtype), "result": torch.stack([norm, c])}
    if s["op"] == "inplace":
        # the tensors are slices of one vector for each type: plain operations take these whole
        wide = [v.float() for v in s["vectors"]]
        norm, c = _plain_factor(torch.stack([v.square().sum().sqrt() for v in wide]), s["max_norm"])
        return {"grads": [v.copy_(w * c) for v, w in zip(s["vectors"], wide)], "result": torch.stack([norm, c])}
    if s["op"] == "server":
        acc = s["grads"][0]
        norm, c = _plain_factor(acc, s["max_norm"])
        s["params"] -= s["lr"] * (c * acc)
        return {"params": s["params"], "result": torch.stack([norm, c])}
    ids = s["ids"].long()
    held = (ids >= 0) & (ids < s["rows"])
    ids = torch.where(held, ids, 0)
    if s["op"] == "lookup":
        y = torch.where(held[:, None], s["table"][ids].float() * s["scale"], 0.0)
        return {"y": y.to(s["y"].dtype)}
    d = torch.where(held[:, None], s["dout"].float() * s["scale"], 0.0)
    if s["add"] and s["grad"].dtype == torch.float32:
        s["grad"].index_add_(0, ids, d)
    else:
        total = torch.zeros(s["grad"].shape, device="cuda").index_add_(0, ids, d)
        s["grad"].copy_(s["grad"].float() + total if s["add"] else total)
    return {"grad": s["grad"]}


def _workspace(s, floats):
    """The scratch memory of a call, which a program keeps from step to step."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(1, floats()), device="cuda")
    return s["workspace"]


def _own(s):
    import paper_1804_08066_b200 as mqg
    if s["op"] in ("flatten", "inplace", "server"):
        w = _workspace(s, lambda: mqg.mqg_norm_workspace_floats(len(s["grads"])))
        if s["op"] == "flatten":
            mqg.mqg_clip_flatten(s["grads"], s["max_norm"], s["flat"], s["result"], w)
            return {"flat": s["flat"], "result": s["result"]}
        if s["op"] == "inplace":
            mqg.mqg_clip_grad_norm(s["grads"], s["max_norm"], s["result"], w)
            return {"grads": s["vectors"], "result": s["result"]}
        acc = s["grads"][0]
        mqg.mqg_grad_norm(s["grads"], s["max_norm"], s["result"], w)
        mqg.mqg_apply_clipped(s["params"], acc, s["lr"], s["result"][1:], acc.numel())
        return {"params": s["params"], "result": s["result"]}
    if s["op"] == "lookup":
        mqg.mqg_embedding(s["table"], s["rows"], s["dim"], s["ids"], s["tokens"], s["scale"], s["y"])
        return {"y": s["y"]}
    w = _workspace(s, lambda: mqg.mqg_embedding_workspace_floats(s["tokens"], s["rows"], s["dim"]))
    mqg.mqg_embedding_grad(s["dout"], s["ids"], s["tokens"], s["rows"], s["dim"], s["scale"], s["grad"], w,
                           add_into_grad=s["add"])
    return {"grad": s["grad"]}


def run(state):
    out = _own(state) if own else _plain(state)
    if state["op"] == "inplace" and state["limit"] < 1:
        state["max_norm"] *= 0.9999      # a limit that tightens from step to step: there is something to clip in each
    return out


def _touched(case):
    """How many rows a batch of ids reaches, on average."""
    k = np.arange(case["rows"], dtype=np.float64)
    if case["spread"] == "zipf":
        p = np.log1p(1.0 / (k + 1.0)) / math.log(max(2, case["rows"]))
    else:
        p = np.full(case["rows"], 1.0 / case["rows"])
    return float((1.0 - np.exp(case["tokens"] * (1.0 - case["empty"]) * np.log1p(-np.minimum(p, 1 - 1e-12)))).sum())


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] in ("flatten", "inplace", "server"):
        sizes = _sizes(case)
        n = sum(sizes)
        read = sum(s * size[k] for s, k in zip(sizes, _kinds(case, len(sizes))))
        if case["op"] == "flatten":
            return {"bytes": read + n * size[case["out"]] + 8, "flops": 3 * n}
        if case["op"] == "server":
            return {"bytes": read + 8 * n + 8, "flops": 5 * n}
        return {"bytes": read + 8 if case["limit"] > 1 else 2 * read + 8, "flops": (2 if case["limit"] > 1 else 3) * n}
    tokens, dim, used = case["tokens"], case["dim"], _touched(case)
    ids = tokens * (8 if case["ids"] == "i64" else 4)
    held = tokens * (1.0 - case["empty"])
    if case["op"] == "lookup":
        return {"bytes": ids + used * dim * size[case["types"]] + tokens * dim * size[case["out"]], "flops": held * dim}
    written = 2 * used if case["add"] else case["rows"]
    return {"bytes": ids + held * dim * size[case["types"]] + written * dim * size[case["out"]], "flops": held * dim}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("flatten", "inplace", "server"):
        total = math.fsum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["grads"])
        norm = math.sqrt(total)
        c = 1.0 if norm <= s["max_norm"] else s["max_norm"] / norm
        result = torch.tensor([norm, c], dtype=torch.float64)
        if case["op"] == "server":
            return {"params": torch.addcmul(s["params"].double(), s["grads"][0].double(), torch.tensor(1.0, device="cuda"),
                                            value=-s["lr"] * c), "result": result}
        if case["op"] == "inplace":
            return {"grads": [v.double().mul_(c) for v in s["vectors"]], "result": result}
        flat = torch.empty(sum(g.numel() for g in s["grads"]), dtype=torch.float64, device="cuda")
        at = 0
        for g in s["grads"]:
            flat[at:at + g.numel()] = g
            at += g.numel()
        return {"flat": flat.mul_(c), "result": result}
    ids = s["ids"].to(torch.int64)
    place = torch.nonzero((ids >= 0) & (ids < case["rows"]))[:, 0]
    if case["op"] == "lookup":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        y[place] = s["table"].double()[ids[place]] * s["scale"]
        return {"y": y}
    grad = s["grad"].double() if case["add"] else torch.zeros(s["grad"].shape, dtype=torch.float64, device="cuda")
    # tokens in the order of their ids: the sum of a row is a difference of running sums
    order = place[torch.argsort(ids[place], stable=True)]
    step = max(1, 2 ** 27 // max(1, order.numel()))
    there, count = torch.unique_consecutive(ids[order], return_counts=True)
    last = torch.cumsum(count, 0) - 1
    for lo in range(0, case["dim"], step):
        run_sum = torch.cumsum(s["dout"][:, lo:lo + step][order].double(), 0)[last]
        grad[there, lo:lo + step] += torch.diff(run_sum, dim=0, prepend=torch.zeros_like(run_sum[:1])) * s["scale"]
    return {"grad": grad}
