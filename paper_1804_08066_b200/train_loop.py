"""The whole MQGrad loop on one GPU with simulated workers (Algorithm 1 end to end):

    python -m paper_1804_08066_b200.train_loop [--iters 60] [--workers 4] [--selector window|sarsa]
                                               [--model cnn|tokens] [--clip C] [--clip-at worker|server]

A small CNN (3x3 convolutions 3-32-64-128, two fully connected layers) is trained on synthetic
32x32x3 images (ten fixed Gaussian class means plus unit noise), batch 128 per worker.  Every
iteration each worker's flat gradient goes through mqg_quantize, the server pass
mqg_server_step updates the shared flat parameter vector, and the host selector picks the next
bit width from the losses.  The model and its autograd belong to this harness; the library is
the codec and what stands around it: with `--model tokens` the model is a classifier of token
sequences (synthetic too: every class prefers some tokens, lengths vary) whose table is looked up
by mqg_embedding and gets its gradient from mqg_embedding_grad; with `--clip C` a worker's
gradients are clipped to norm C on their way into the flat vector (mqg_clip_flatten), or the
server measures the mean of the decoded gradients and applies it clipped (mqg_grad_norm,
mqg_apply_clipped).  Prints one JSON line with the share of iteration time spent inside libmqgrad
(the paper's Table 3 reports 4.1-13.3 % for quantize + de-quantize + MDP on its CPU clusters).
"""
from __future__ import annotations

import argparse
import contextlib
import json
import time

import torch
import torch.nn as nn
import torch.nn.functional as F

import paper_1804_08066_b200 as mqg
from paper_1804_08066_b200.selector import SarsaBitSelector, WindowQSelector

BUCKET = 2048
# Table 3 of the paper: smallest and largest share of training time (%) spent in quantize +
# de-quantize + MDP over its two CPU clusters and five methods; quoted as context in the report.
PAPER_TABLE_3_RANGE_PERCENT = (4.11, 13.3)


class SmallCnn(nn.Module):
    def __init__(self):
        super().__init__()
        self.c1 = nn.Conv2d(3, 32, 3, padding=1)
        self.c2 = nn.Conv2d(32, 64, 3, padding=1)
        self.c3 = nn.Conv2d(64, 128, 3, padding=1)
        self.f1 = nn.Linear(128 * 4 * 4, 256)
        self.f2 = nn.Linear(256, 10)

    def forward(self, x):
        x = F.max_pool2d(F.relu(self.c1(x)), 2)
        x = F.max_pool2d(F.relu(self.c2(x)), 2)
        x = F.max_pool2d(F.relu(self.c3(x)), 2)
        return self.f2(F.relu(self.f1(x.flatten(1))))


VOCABULARY, WIDTH, LENGTH = 1000, 64, 16         # tokens, elements of a table's row, places of a sequence


class TokenClassifier(nn.Module):
    """The mean of a sequence's table rows (times sqrt(WIDTH)), and two fully connected layers."""

    scale = WIDTH ** 0.5

    def __init__(self):
        super().__init__()
        self.table = nn.Parameter(torch.randn(VOCABULARY, WIDTH) / WIDTH)
        self.f1 = nn.Linear(WIDTH, 128)
        self.f2 = nn.Linear(128, 10)

    def forward(self, rows, held):
        """`rows`: the scaled table rows of [batch, LENGTH] places, zero in the empty ones; `held`: which are not empty."""
        mean = rows.sum(1) / held.sum(1, keepdim=True).clamp(min=1)
        return self.f2(F.relu(self.f1(mean)))


def token_batch(gen, batch):
    """Ids [batch, LENGTH] with -1 behind a sequence's end, and labels; a class draws every second token from its own tenth of
    the vocabulary."""
    y = torch.randint(0, 10, (batch,), generator=gen, device="cuda")
    own = y[:, None] + 10 * torch.randint(0, VOCABULARY // 10, (batch, LENGTH), generator=gen, device="cuda")
    ids = torch.randint(0, VOCABULARY, (batch, LENGTH), generator=gen, device="cuda")
    ids = torch.where(torch.rand(batch, LENGTH, generator=gen, device="cuda") < 0.5, own, ids)
    length = torch.randint(1, LENGTH + 1, (batch, 1), generator=gen, device="cuda")
    return torch.where(torch.arange(LENGTH, device="cuda") < length, ids, -1), y


def token_gradients(model, ids, y, workspace, library=contextlib.nullcontext()):
    """Loss of a batch and the gradient of every parameter, in their order; the library's calls run within `library`."""
    n = ids.numel()
    rows = torch.empty(*ids.shape, WIDTH, device="cuda")
    with library:
        mqg.mqg_embedding(model.table.data, VOCABULARY, WIDTH, ids, n, model.scale, rows)
    rows.requires_grad_()
    model.zero_grad(set_to_none=True)
    loss = F.cross_entropy(model(rows, ids >= 0), y)
    loss.backward()
    table = torch.empty_like(model.table.data)
    dout = rows.grad.contiguous()
    with library:
        mqg.mqg_embedding_grad(dout, ids, n, VOCABULARY, WIDTH, model.scale, table, workspace)
    return loss, [table, *(p.grad for p in model.parameters() if p is not model.table)]


class LibraryTime:
    """Device time of the library's work: the time between the events around each `with` block."""

    def __init__(self):
        self.spans = []

    def __enter__(self):
        self.spans.append([torch.cuda.Event(enable_timing=True) for _ in range(2)])
        self.spans[-1][0].record()

    def __exit__(self, *_):
        self.spans[-1][1].record()

    def take(self):
        """Milliseconds since the last call of this; the device must have finished the blocks."""
        ms = sum(a.elapsed_time(b) for a, b in self.spans)
        self.spans.clear()
        return ms


def flatten_parameters(model):
    """Re-seat every parameter as a view into one flat fp32 vector (the shared parameters w)."""
    n = sum(p.numel() for p in model.parameters())
    flat = torch.zeros(n, dtype=torch.float32, device="cuda")
    off = 0
    for p in model.parameters():
        flat[off:off + p.numel()].copy_(p.data.reshape(-1))
        p.data = flat[off:off + p.numel()].view_as(p.data)
        off += p.numel()
    return flat


def run(iters=60, workers=4, batch=128, lr=0.05, selector="window", seed=0, model="cnn", clip=None, clip_at="worker"):
    torch.manual_seed(seed)
    kind, model = model, (SmallCnn() if model == "cnn" else TokenClassifier()).cuda()
    flat = flatten_parameters(model)
    n = flat.numel()
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    if kind == "cnn":
        means = torch.randn(10, 3, 32, 32, generator=gen, device="cuda")
    else:
        sums = torch.empty(mqg.mqg_embedding_workspace_floats(batch * LENGTH, VOCABULARY, WIDTH), device="cuda")
    norms = torch.zeros(iters, workers if clip_at == "worker" else 1, 2, device="cuda")       # norm and factor
    norm_workspace = torch.empty(mqg.mqg_norm_workspace_floats(len(list(model.parameters()))), device="cuda")
    acc = torch.empty(n, device="cuda") if clip is not None and clip_at == "server" else None
    sel = WindowQSelector(seed=seed) if selector == "window" else SarsaBitSelector(seed=seed)
    codes = [torch.zeros(mqg.mqg_code_words(n, 8), dtype=torch.int32, device="cuda") for _ in range(workers)]
    scales = [torch.zeros(mqg.mqg_num_buckets(n, BUCKET), dtype=torch.float32, device="cuda") for _ in range(workers)]
    bits, lib_ms, total_ms, wire = (1 if selector == "window" else 2), 0.0, 0.0, 0
    losses, chosen, library = [], [], LibraryTime()
    last_ms = 1.0
    for m in range(iters):
        t0 = time.perf_counter()
        torch.cuda.synchronize()
        grads, loss_sum = [], 0.0
        for w in range(workers):
            if kind == "cnn":
                y = torch.randint(0, 10, (batch,), generator=gen, device="cuda")
                x = means[y] + torch.randn(batch, 3, 32, 32, generator=gen, device="cuda")
                model.zero_grad(set_to_none=True)
                loss = F.cross_entropy(model(x), y)
                loss.backward()
                parts = [p.grad for p in model.parameters()]
            else:
                loss, parts = token_gradients(model, *token_batch(gen, batch), sums, library)
            if clip is not None and clip_at == "worker":
                grads.append(torch.empty(n, device="cuda"))
                parts = [g.contiguous() for g in parts]
                with library:
                    mqg.mqg_clip_flatten(parts, clip, grads[w], norms[m, w], norm_workspace)
            else:
                grads.append(torch.cat([g.reshape(-1) for g in parts]))
            loss_sum += float(loss.detach())
        loss_m = loss_sum / workers
        bits = sel.step(m, loss_m, last_ms)                       # server MDP: loss in, width out
        with library:
            for w in range(workers):
                mqg.mqg_quantize(grads[w], n, bits, BUCKET, seed, codes[w], scales[w], worker=w, step=m)
            if acc is None:
                mqg.mqg_server_step(codes, scales, workers, bits, n, BUCKET, flat, lr / workers)
            else:                                                 # the mean's norm is the sum's / workers
                mqg.mqg_dequant_accumulate(codes, scales, workers, bits, n, acc, BUCKET)
                mqg.mqg_grad_norm([acc], clip * workers, norms[m, 0], norm_workspace)
                mqg.mqg_apply_clipped(flat, acc, lr / workers, norms[m, 0, 1:], n)
        torch.cuda.synchronize()
        lib_ms += library.take()
        last_ms = (time.perf_counter() - t0) * 1e3
        total_ms += last_ms
        wire += workers * mqg.mqg_wire_bytes(n, bits, BUCKET)
        losses.append(loss_m), chosen.append(bits)
    assert mqg.mqg_device_timeouts() == 0
    return {"iters": iters, "workers": workers, "parameters": n, "selector": selector, "model": kind,
            "clip_norm": clip, "clip_factors": None if clip is None else norms[..., 1].mean(1).tolist(),
            "first_loss": losses[0], "last_loss": losses[-1], "bits_chosen": chosen,
            "libmqgrad_ms_per_iter": lib_ms / iters, "iteration_ms": total_ms / iters,
            "libmqgrad_share_pct": 100.0 * lib_ms / total_ms,
            "uplink_bytes_per_iter": wire / iters, "uplink_bytes_fp32": 4 * n * workers,
            "paper_table3_share_pct": "%g-%g (CPU clusters, quantize + de-quantize + MDP)"
                                      % PAPER_TABLE_3_RANGE_PERCENT}


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--iters", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--selector", default="window", choices=["window", "sarsa"])
    ap.add_argument("--model", default="cnn", choices=["cnn", "tokens"])
    ap.add_argument("--clip", type=float, default=None, help="largest norm of a gradient")
    ap.add_argument("--clip-at", default="worker", choices=["worker", "server"])
    a = ap.parse_args()
    print(json.dumps(run(a.iters, a.workers, selector=a.selector, model=a.model, clip=a.clip, clip_at=a.clip_at)))
