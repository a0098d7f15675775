"""The loop with AdamW and with the layer norm: that it runs, its gradients against 64-bit autograd, and one iteration by hand."""
import math

import numpy as np
import pytest
import torch
import torch.nn.functional as F

import paper_1804_08066_b200 as mqg

from .adamw_plain import step64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("model,norm", [("cnn", False), ("tokens", False), ("tokens", True)])
@pytest.mark.parametrize("optimizer", ["sgd", "adamw", "adamw8"])
@pytest.mark.parametrize("clip_at", [None, "worker", "server"])
def test_the_loop_runs(model, norm, optimizer, clip_at):
    from paper_1804_08066_b200.train_loop import run
    r = run(iters=4, workers=3, batch=32, seed=2, model=model, norm=norm, optimizer=optimizer, clip=clip_at and 0.05, clip_at=clip_at or "worker")
    assert math.isfinite(r["last_loss"]) and r["optimizer"] == optimizer and r["norm"] == norm
    assert r["parameters"] == (620_362 if model == "cnn" else 1000 * 64 + 128 * norm + 64 * 128 + 128 + 1290)
    if clip_at:
        assert all(0 < f < 1 for f in r["clip_factors"])


@pytest.mark.parametrize("optimizer,norm", [("adamw", True), ("adamw8", False)])
def test_the_library_share_counts_every_call_into_the_library(monkeypatch, optimizer, norm):
    from paper_1804_08066_b200 import train_loop as tl
    recorded, calls = [0], []
    record = torch.cuda.Event.record

    def count(self, *args, **kwargs):
        recorded[0] += 1
        return record(self, *args, **kwargs)

    class Watched:
        def __getattr__(self, name):
            value = getattr(mqg, name)
            if name not in mqg._NATIVE and name not in mqg._NATIVE_AROUND:
                return value

            def call(*args, **kwargs):
                calls.append((name, recorded[0] % 2 == 1))
                return value(*args, **kwargs)
            return call

    monkeypatch.setattr(torch.cuda.Event, "record", count)
    monkeypatch.setattr(tl, "mqg", Watched())
    tl.run(iters=2, workers=2, batch=32, model="tokens", norm=norm, optimizer=optimizer)
    want = {"mqg_quantize", "mqg_embedding", "mqg_embedding_grad", "mqg_dequant_accumulate", "mqg_" + optimizer}
    assert {name for name, _ in calls} == want | ({"mqg_layer_norm", "mqg_layer_norm_grad"} if norm else set())
    assert [name for name, timed in calls if not timed] == []


def test_gradients_of_the_normalised_token_model():
    """Sums of at most 512 terms (batch 32, 16 places) through eight products and the norm's own sums of 64: 16 * 512 * 2^-24 of the
    largest gradient of a tensor, above all the roundings on the way."""
    from paper_1804_08066_b200 import train_loop as tl
    torch.manual_seed(0)
    model = tl.TokenClassifier(norm=True).cuda()
    gen = torch.Generator(device="cuda").manual_seed(1)
    with torch.no_grad():
        model.gain.normal_(1.0, 0.2, generator=gen)
        model.shift.normal_(0.0, 0.2, generator=gen)
    ids, y = tl.token_batch(gen, 32)
    assert (ids == -1).any()
    loss, grads = tl.token_gradients(model, ids, y, tl.token_workspace(ids.numel()))

    wide = tl.TokenClassifier(norm=True).double()
    wide.load_state_dict({k: v.double().cpu() for k, v in model.state_dict().items()})
    held = (ids >= 0).cpu()
    rows = torch.where(held[..., None], wide.table[ids.clamp(min=0).cpu()] * wide.scale, 0.0)
    centred = rows - rows.mean(-1, keepdim=True)
    normed = centred / (centred.square().mean(-1, keepdim=True) + wide.eps).sqrt() * wide.gain + wide.shift
    want = F.cross_entropy(wide(normed, held), y.cpu())
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 512 * 2.0 ** -24 * 4
    assert len(grads) == len(list(wide.parameters()))
    for g, p in zip(grads, wide.parameters()):
        assert g.shape == p.shape
        assert (g.double().cpu() - p.grad).abs().max() <= 16 * 512 * 2.0 ** -24 * p.grad.abs().max()


def test_gradients_are_the_same_while_a_graph_of_them_is_captured():
    """The operators have no part in autograd: a captured chain of them beside an eager graph of the same leaves."""
    from paper_1804_08066_b200 import train_loop as tl
    torch.manual_seed(0)
    model = tl.TokenClassifier(norm=True).cuda()
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids, y = tl.token_batch(gen, 16)
    work = tl.token_workspace(ids.numel())
    eager_loss, eager = tl.token_gradients(model, ids, y, work)
    n = ids.numel()
    rows, inner, stats = torch.empty(n, tl.WIDTH, device="cuda"), torch.empty(n, tl.WIDTH, device="cuda"), torch.empty(n, 2, device="cuda")
    drows, dgain, dshift = torch.empty_like(rows), torch.empty(tl.WIDTH, device="cuda"), torch.empty(tl.WIDTH, device="cuda")
    dy = torch.randn(n, tl.WIDTH, device="cuda", generator=gen)
    kept = (eager_loss * 2.0, model(inner.view(*ids.shape, tl.WIDTH).clone().requires_grad_(), ids >= 0))       # a live eager graph

    def chain():
        mqg.mqg_embedding(model.table.data, tl.VOCABULARY, tl.WIDTH, ids, n, model.scale, rows)
        mqg.mqg_layer_norm(rows, n, tl.WIDTH, model.gain.data, model.shift.data, model.eps, inner, stats)
        mqg.mqg_layer_norm_grad(dy, rows, n, tl.WIDTH, model.gain.data, stats, drows, dgain, dshift, work)

    chain()
    want = [t.clone() for t in (inner, drows, dgain, dshift)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for t in (inner, drows, dgain, dshift):
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, (inner, drows, dgain, dshift)))
    kept[1].sum().backward()


def test_norm_gradient_codec_and_adamw_together():
    """One iteration by hand: rows normalised, their gradient, the codec, and the server's AdamW step, against the plain forms."""
    rows, dim, bits, bucket = 300, 72, 8, 256
    gen = torch.Generator().manual_seed(5)
    x, dy = torch.randn(rows, dim, generator=gen) + 0.5, torch.randn(rows, dim, generator=gen) * 1e-2
    params = torch.cat([1 + 0.1 * torch.randn(dim, generator=gen), 0.1 * torch.randn(dim, generator=gen)]).cuda()
    weight, bias = params.split(dim)
    y, stats = torch.empty(rows, dim, device="cuda"), torch.empty(rows, 2, device="cuda")
    mqg.mqg_layer_norm(x.cuda(), rows, dim, weight, bias, 1e-5, y, stats)
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    work = torch.empty(mqg.mqg_layer_norm_workspace_floats(rows, dim), device="cuda")
    mqg.mqg_layer_norm_grad(dy.cuda(), x.cuda(), rows, dim, weight, stats, None, dw, db, work)
    flat, result = torch.empty(2 * dim, device="cuda"), torch.empty(2, device="cuda")
    norm_work = torch.empty(mqg.mqg_norm_workspace_floats(2), device="cuda")
    mqg.mqg_clip_flatten([dw, db], 0.5, flat, result, norm_work)
    codes = torch.zeros(mqg.mqg_code_words(2 * dim, bits), dtype=torch.int32, device="cuda")
    scales = torch.zeros(1, device="cuda")
    mqg.mqg_quantize(flat, 2 * dim, bits, bucket, 9, codes, scales)
    acc = torch.empty(2 * dim, device="cuda")
    mqg.mqg_dequant_accumulate([codes], [scales], 1, bits, 2 * dim, acc, bucket)
    before = params.clone()
    m, v = torch.zeros(2 * dim, device="cuda"), torch.zeros(2 * dim, device="cuda")
    mqg.mqg_grad_norm([acc], 0.25, result, norm_work)
    parts = lambda t: list(t.split(dim))  # noqa: E731
    mqg.mqg_adamw(parts(params), parts(acc), parts(m), parts(v), [0.1, 0.0], 1e-2, 0.9, 0.999, 1e-8, 1, factor=result[1:])

    d = x.double() - x.double().mean(1, keepdim=True)
    h = d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt()
    whole = torch.cat([(dy.double() * h).sum(0), dy.double().sum(0)])
    clipped = whole * min(1.0, 0.5 / float(whole.norm()))
    # a step of the codec's grid is 2 s / 255 of the largest magnitude s; fp32 errors are far below it
    assert ((acc.double().cpu() - clipped).abs() <= 1.001 * 2 * float(clipped.abs().max()) / 255).all()
    wire = acc.cpu().double().numpy()
    k = min(1.0, 0.25 / float(np.linalg.norm(wire)))
    for at, decay in ((slice(0, dim), float(np.float32(0.1))), (slice(dim, 2 * dim), 0.0)):
        want, _, _, slack = step64(before.cpu().numpy()[at], wire[at], np.zeros(dim), np.zeros(dim), lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8,
                                   step=1, decay=decay, k=k)
        # the factor is off by 8 * 2^-24 of itself, which m and the root of v have in common but for eps
        off = np.abs(params.cpu().double().numpy()[at] - want)
        assert (off <= slack + 8 * 2.0 ** -24 * 1e-2).all()
