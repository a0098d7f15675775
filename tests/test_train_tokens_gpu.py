"""The loop with a table over tokens and with clipping: that it runs, and its gradients against 64-bit autograd."""
import math

import pytest
import torch
import torch.nn.functional as F

import paper_1804_08066_b200 as mqg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("model", ["cnn", "tokens"])
@pytest.mark.parametrize("clip,clip_at", [(None, "worker"), (0.05, "worker"), (0.05, "server"), (1e6, "server")])
def test_the_loop_runs_with_each_model_and_clip(model, clip, clip_at):
    from paper_1804_08066_b200.train_loop import run
    r = run(iters=6, workers=3, batch=32, seed=2, model=model, clip=clip, clip_at=clip_at)
    assert r["model"] == model and math.isfinite(r["last_loss"])
    assert r["parameters"] == (620_362 if model == "cnn" else 1000 * 64 + 64 * 128 + 128 + 1290)
    if clip is None:
        assert r["clip_factors"] is None
    else:
        assert len(r["clip_factors"]) == 6 and all(0 < f <= 1 for f in r["clip_factors"])
        assert all((f == 1) == (clip == 1e6) for f in r["clip_factors"])


@pytest.mark.parametrize("model,clip,clip_at", [("cnn", None, "worker"), ("cnn", 0.05, "worker"), ("tokens", 0.05, "worker"),
                                                ("tokens", 0.05, "server")])
def test_the_library_share_counts_every_call_into_the_library(monkeypatch, model, clip, clip_at):
    """Events are recorded in pairs around what is timed: every call that enqueues work stands between the two of one."""
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
    r = tl.run(iters=2, workers=2, batch=32, model=model, clip=clip, clip_at=clip_at)
    want = {"mqg_quantize"} | ({"mqg_embedding", "mqg_embedding_grad"} if model == "tokens" else set())
    if clip is None:
        want |= {"mqg_server_step"}
    elif clip_at == "worker":
        want |= {"mqg_server_step", "mqg_clip_flatten"}
    else:
        want |= {"mqg_dequant_accumulate", "mqg_grad_norm", "mqg_apply_clipped"}
    assert {name for name, _ in calls} == want
    assert [name for name, timed in calls if not timed] == []
    assert recorded[0] % 2 == 0 and 0 < r["libmqgrad_share_pct"] < 100


def test_a_limit_that_nothing_reaches_changes_nothing():
    from paper_1804_08066_b200.train_loop import run
    plain, limited = (run(iters=4, workers=2, batch=32, seed=3, model="tokens", clip=c) for c in (None, 1e6))
    assert plain["first_loss"] == limited["first_loss"] and plain["last_loss"] == limited["last_loss"]


def test_gradients_of_the_token_model():
    """Every step up to the last layers is linear in fp32; the bound is the accumulated relative error of sums of at most 512
    terms (batch 32, 16 places) through four products, 4 * 512 * 2^-24 of the largest gradient of a tensor."""
    from paper_1804_08066_b200 import train_loop as tl
    torch.manual_seed(0)
    model = tl.TokenClassifier().cuda()
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids, y = tl.token_batch(gen, 32)
    assert (ids == -1).any() and (ids.max() < tl.VOCABULARY)
    work = torch.empty(mqg.mqg_embedding_workspace_floats(ids.numel(), tl.VOCABULARY, tl.WIDTH), device="cuda")
    loss, grads = tl.token_gradients(model, ids, y, work)

    wide = tl.TokenClassifier().double()
    wide.load_state_dict({k: v.double().cpu() for k, v in model.state_dict().items()})
    held = (ids >= 0).cpu()
    rows = torch.where(held[..., None], wide.table[ids.clamp(min=0).cpu()] * wide.scale, 0.0)
    want = F.cross_entropy(wide(rows, held), y.cpu())
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 512 * 2.0 ** -24 * 4
    for g, p in zip(grads, wide.parameters()):
        assert g.shape == p.shape
        assert (g.double().cpu() - p.grad).abs().max() <= 4 * 512 * 2.0 ** -24 * p.grad.abs().max()


def test_lookup_gradient_clip_codec_and_update_together():
    """One iteration of a worker and the server by hand, each step against its plain form."""
    rows, dim, tokens, bits, bucket, lr = 700, 40, 900, 8, 256, 0.25
    gen = torch.Generator().manual_seed(5)
    table = torch.randn(rows, dim, generator=gen)
    ids = torch.randint(-5, rows, (tokens,), generator=gen)
    dout = torch.randn(tokens, dim, generator=gen) * 1e-2
    bias = torch.randn(17, generator=gen)
    n = rows * dim + 17
    params = torch.cat([table.flatten(), torch.zeros(17)]).cuda()
    grads = [torch.empty(rows, dim, device="cuda"), bias.cuda()]
    work = torch.empty(mqg.mqg_embedding_workspace_floats(tokens, rows, dim), device="cuda")
    mqg.mqg_embedding_grad(dout.cuda(), ids.cuda(), tokens, rows, dim, 3.0, grads[0], work)
    flat, result = torch.empty(n, device="cuda"), torch.empty(2, device="cuda")
    norm_work = torch.empty(mqg.mqg_norm_workspace_floats(2), device="cuda")
    mqg.mqg_clip_flatten(grads, 0.5, flat, result, norm_work)
    codes = torch.zeros(mqg.mqg_code_words(n, bits), dtype=torch.int32, device="cuda")
    scales = torch.zeros(mqg.mqg_num_buckets(n, bucket), device="cuda")
    mqg.mqg_quantize(flat, n, bits, bucket, 9, codes, scales)
    acc = torch.empty(n, device="cuda")
    mqg.mqg_dequant_accumulate([codes], [scales], 1, bits, n, acc, bucket)
    before = params.clone()
    mqg.mqg_grad_norm([acc], 0.25, result[:2], norm_work)
    mqg.mqg_apply_clipped(params, acc, lr, result[1:], n)
    out = torch.empty(tokens, dim, device="cuda")
    mqg.mqg_embedding(params[:rows * dim], rows, dim, ids.cuda(), tokens, 1.0, out)

    held = ids >= 0
    g = torch.zeros(rows, dim, dtype=torch.float64).index_add_(0, ids[held], dout[held].double()) * 3.0
    whole = torch.cat([g.flatten(), bias.double()])
    clipped = whole * min(1.0, 0.5 / float(whole.norm()))
    # one step of the codec's grid is 2 s / 255 of the bucket's largest magnitude s; fp32 errors are far below it
    step = torch.cat([torch.full_like(c, 2 * float(c.abs().max()) / 255) for c in clipped.split(bucket)])
    assert ((acc.double().cpu() - clipped).abs() <= 1.001 * step + 1e-12).all()
    wire = acc.double().cpu()
    moved = before.double().cpu() - float(torch.tensor(lr)) * min(1.0, 0.25 / float(wire.norm())) * wire
    # the factor is off by 8 * 2^-24 of itself, and there are roundings of the product and of the sum
    assert ((params.double().cpu() - moved).abs() <= 2.0 ** -24 * (11 * lr * wire.abs() + 1.01 * moved.abs())).all()
    want = torch.zeros(tokens, dim)
    want[held] = params.cpu()[:rows * dim].view(rows, dim)[ids[held]]
    assert torch.equal(out.cpu(), want)
