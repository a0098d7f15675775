"""Tensors of a call live until it has returned, also where another thread empties its lists while it runs without the interpreter
lock: here a call that waits for room in a full launch queue."""
import threading
import time
import weakref

import pytest
import torch

import paper_1804_08066_b200 as mqg

pytestmark = pytest.mark.gpu


def zeros(count, n=64, dtype=torch.float32):
    return [torch.zeros(n, dtype=dtype, device="cuda") for _ in range(count)]


def adamw():
    lists = [zeros(3) for _ in range(4)]
    return lists, lambda: mqg.mqg_adamw(*lists, None, 1e-3, 0.9, 0.999, 1e-8, 1)


def adamw8():
    lists = [zeros(3), zeros(3), zeros(3, dtype=torch.uint8), zeros(3, dtype=torch.uint8), zeros(3, 2)]
    return lists, lambda: mqg.mqg_adamw8(*lists, None, 1e-3, 0.9, 0.999, 1e-8, 1, 7)


def grad_norm():
    grads, result = zeros(3), torch.zeros(2, device="cuda")
    work = torch.zeros(mqg.mqg_norm_workspace_floats(3), device="cuda")
    return [grads], lambda: mqg.mqg_grad_norm(grads, 1.0, result, work)


def quantize_workers():
    grads, codes, scales = zeros(3, 4096), zeros(3, mqg.mqg_code_words(4096, 4), torch.int32), zeros(3, mqg.mqg_num_buckets(4096, 2048))
    return [grads, codes, scales], lambda: mqg.mqg_quantize_workers(grads, 3, 4096, 4, 2048, 1, codes, scales)


@pytest.mark.parametrize("make", [adamw, adamw8, grad_norm, quantize_workers])
def test_lists_emptied_while_a_call_waits(make):
    lists, call = make()
    call()
    torch.cuda.synchronize()
    refs = [weakref.ref(t) for x in lists for t in x]
    seen = {}

    def empty_them():
        time.sleep(0.4)                                 # by now the queue is full
        seen["calls"] = count
        for x in lists:
            x.clear()
        seen["alive"] = sum(r() is not None for r in refs)

    count, refused = 0, False
    other = threading.Thread(target=empty_them)
    torch.cuda._sleep(2_500_000_000)                    # more than a second
    other.start()
    try:
        for count in range(1, 20_000):
            call()
    except (ValueError, IndexError, TypeError):         # the next call finds its lists empty
        refused = True
    other.join()
    after = sum(r() is not None for r in refs)
    torch.cuda.synchronize()
    # adamw and grad_norm of no tensors are calls like any other
    assert refused or make in (adamw, adamw8, grad_norm)
    assert 0 < seen["calls"] < 19_999, "the queue was never full"
    assert seen["alive"] == len(refs) and after == 0
    assert mqg.mqg_device_timeouts() == 0
