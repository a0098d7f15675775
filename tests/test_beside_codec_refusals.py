"""Calls of the AdamW and layer norm operators that are refused before anything reaches the device, and what their sources have to
hold.  No GPU needed: the C ABI checks its arguments on the host, the binding its tensors."""
import ctypes as C
import math
import re

import pytest
import torch

import paper_1804_08066_b200 as mqg

from .test_launch_waits import CSRC, _bodies

OK, INVALID, ALIGN = mqg.MQG_OK, mqg.MQG_ERR_INVALID, mqg.MQG_ERR_ALIGN
P = 0x100000                                             # never dereferenced on the host
FLOATS = 1 << 24


@pytest.fixture(scope="module")
def lib():
    return mqg.raw_library()


def pointers(*p):
    return (C.c_void_p * len(p))(*p)


def lists(eight, sizes=(100, 7), **put):
    """Arguments up to `count`; tensor j of list k lies at P + (k * 8 + j) * 65536."""
    n = len(sizes)
    at = {k: [P + (i * 8 + j) * 65536 for j in range(n)] for i, k in enumerate(("p", "g", "m", "v", "s"))}
    types = {"pt": [0] * n, "gt": [1] * n}
    decays = [0.1] * n
    for name, (j, value) in put.items():
        (decays if name == "d" else types[name] if name in types else at[name])[j] = value
    head = [pointers(*at["p"]), (C.c_int * n)(*types["pt"]), pointers(*at["g"]), (C.c_int * n)(*types["gt"]), pointers(*at["m"]),
            pointers(*at["v"])]
    tail = [(C.c_uint64 * n)(*sizes), (C.c_float * n)(*decays), n]
    return head + ([pointers(*at["s"])] if eight else []) + tail


def call(lib, eight, args, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, step=1, scale=1.0, factor=None, schedule=None):
    if eight:
        return lib.mqg_adamw8(*args, lr, b1, b2, eps, step, 3, scale, factor, schedule, None)
    return lib.mqg_adamw(*args, lr, b1, b2, eps, step, scale, factor, schedule, None)


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_numbers_of_adamw_are_checked(lib, eight):
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(b1=1.0), dict(b1=-0.1), dict(b1=math.nan), dict(b2=1.0),
                dict(b2=1 - 1e-9), dict(eps=0.0), dict(eps=1e-17), dict(eps=math.inf), dict(eps=math.nan), dict(scale=math.inf),
                dict(scale=math.nan), dict(step=0)):
        assert call(lib, eight, lists(eight), **bad) == INVALID, bad
    assert call(lib, eight, lists(eight), factor=P + 2) == ALIGN
    assert call(lib, eight, lists(eight), schedule=P + 1, step=0) == ALIGN


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_lists_of_adamw_are_checked(lib, eight):
    for name in "pgmv" + "s" * eight:
        assert call(lib, eight, lists(eight, **{name: (1, None)})) == INVALID and "tensor 1 is null" in mqg.mqg_last_error()
        if not (eight and name in "mv"):                 # (bytes lie anywhere: that call would run)
            assert call(lib, eight, lists(eight, **{name: (0, P + (1 << 30) + 1)})) == ALIGN, name
    for bad in (dict(pt=(0, 2)), dict(gt=(1, -1)), dict(d=(0, -1.0)), dict(d=(1, math.nan)), dict(d=(1, math.inf))):
        assert call(lib, eight, lists(eight, **bad)) == INVALID, bad
    assert call(lib, eight, lists(eight, sizes=(1 << 42,))) == INVALID
    assert call(lib, eight, lists(eight, sizes=(1 << 41, 1 << 41))) == INVALID
    good = lists(eight)
    for k in range(len(good) - 1):
        if good[k] is not good[-2]:                      # decays may be left out
            assert call(lib, eight, good[:k] + [None] + good[k + 1:]) == INVALID, k
    assert call(lib, eight, good[:-1] + [-1]) == INVALID
    assert call(lib, eight, [None] * (len(good) - 1) + [0]) == OK
    empty = lists(eight, sizes=(0, 0), p=(0, None), m=(1, None))
    assert call(lib, eight, empty) == OK


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_memory_that_adamw_shares_is_refused(lib, eight):
    names = "pgmv" + "s" * eight
    where = {k: P + i * 8 * 65536 for i, k in enumerate(names)}
    for a in names:
        for b in names:
            if a != b:
                assert call(lib, eight, lists(eight, **{a: (1, where[b])})) == INVALID and "share memory" in mqg.mqg_last_error(), a + b
        if a != "g":
            assert call(lib, eight, lists(eight, **{a: (1, where[a])})) == INVALID and "share memory" in mqg.mqg_last_error(), a
            assert call(lib, eight, lists(eight), factor=where[a] + 4) == INVALID
            assert call(lib, eight, lists(eight), schedule=where[a] - 12) == INVALID
    # the last byte of one and the first of the next; lists out of order, where the pieces are sorted
    down = lists(eight, sizes=(8, 8, 8), p=(0, P + 3 * 65536))
    assert call(lib, eight, [*down[:-1], 3], factor=P + 65536 + 28) == INVALID


def test_rows_of_layer_norm_are_checked(lib):
    def norm(x=P, xt=0, rows=4, dim=8, w=P + 4096, b=P + 8192, wt=0, eps=1e-5, y=P + 12288, yt=0, stats=P + 16384):
        return lib.mqg_layer_norm(x, xt, rows, dim, w, b, wt, eps, y, yt, stats, None)
    for bad in (dict(x=None), dict(y=None), dict(xt=2), dict(yt=-1), dict(wt=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan),
                dict(eps=math.inf), dict(rows=1 << 31), dict(dim=(1 << 22) + 1), dict(rows=0, eps=0.0)):
        assert norm(**bad) == INVALID, bad
    for bad in (dict(x=P + 2), dict(y=P + 12289, yt=1), dict(w=P + 4098), dict(b=P + 8194), dict(stats=P + 16385)):
        assert norm(**bad) == ALIGN, bad
    for bad in (dict(y=P), dict(y=P + 124), dict(stats=P + 124), dict(stats=P + 12288), dict(y=P + 4096), dict(b=P + 12288 + 64),
                dict(stats=P + 4096 + 28)):
        assert norm(**bad) == INVALID and "share memory" in mqg.mqg_last_error(), bad
    assert norm(rows=0, x=None, y=None) == OK and norm(dim=0, x=None, y=None, w=None, b=None, stats=None) == OK


def test_layer_norm_gradients_are_checked(lib):
    def grad(dy=P, dyt=0, x=P + 4096, xt=0, rows=4, dim=8, w=P + 8192, wt=0, stats=P + 12288, dx=P + 16384, dw=P + 20480,
             db=P + 24576, dwt=0, add=0, work=P + (1 << 20), floats=FLOATS):
        return lib.mqg_layer_norm_grad(dy, dyt, x, xt, rows, dim, w, wt, stats, dx, dw, db, dwt, add, work, floats, None)
    for bad in (dict(dy=None), dict(x=None), dict(stats=None), dict(dyt=2), dict(xt=-1), dict(wt=2), dict(dwt=9), dict(rows=1 << 31),
                dict(dim=(1 << 22) + 1), dict(work=None), dict(floats=mqg.mqg_layer_norm_workspace_floats(4, 8) - 1)):
        assert grad(**bad) == INVALID, bad
    for bad in (dict(dy=P + 2), dict(x=P + 4097, xt=1), dict(w=P + 8193), dict(stats=P + 12290), dict(dx=P + 16386),
                dict(dw=P + 20482), dict(db=P + 24577, dwt=1), dict(work=P + (1 << 20) + 8)):
        assert grad(**bad) == ALIGN, bad
    for bad in (dict(dx=P), dict(dx=P + 4096), dict(dx=P + 12288), dict(dw=P + 8192), dict(db=P + 20480 + 28), dict(dw=P + 16384 + 124),
                dict(db=P + 124), dict(work=P), dict(work=P + 4096), dict(work=P + 8192), dict(work=P + 12288), dict(work=P + 24576)):
        assert grad(**bad) == INVALID and "share memory" in mqg.mqg_last_error(), bad
    assert grad(dx=None, dw=None, db=None) == OK and grad(rows=0, dy=None, x=None, stats=None, add=1) == OK
    assert grad(dim=0, dy=None, x=None, stats=None, w=None) == OK
    assert mqg.mqg_layer_norm_workspace_floats(1 << 31, 8) == 0 == mqg.mqg_layer_norm_workspace_floats(8, (1 << 22) + 1)


def test_scale_floats():
    assert [mqg.mqg_adamw8_scale_floats(n) for n in (0, 1, 256, 257, 1 << 40)] == [0, 2, 2, 4, 1 << 33]


def test_the_binding_refuses_what_it_cannot_take():
    t = torch.zeros(8)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    with pytest.raises(TypeError, match="CUDA tensor"):
        mqg.mqg_adamw([t], [t], [t], [t], 0.0, **hyper)
    with pytest.raises(ValueError, match="m holds 2 tensors, params 1"):
        mqg.mqg_adamw([t], [t], [t, t], [t], 0.0, **hyper)
    with pytest.raises(ValueError, match="decays holds 2 numbers"):
        mqg.mqg_adamw([t], [t], [t], [t], [0.0, 0.1], **hyper)
    with pytest.raises(TypeError):
        mqg.mqg_adamw(3, [t], [t], [t], 0.0, **hyper)
    with pytest.raises(TypeError):
        mqg.mqg_adamw([t], [t], [t], [t], "x", **hyper)
    with pytest.raises(ValueError, match="step"):
        mqg.mqg_adamw([t], [t], [t], [t], 0.0, **{**hyper, "step": 1 << 32})
    with pytest.raises(TypeError, match="CUDA tensor"):
        mqg.mqg_adamw8([t], [t], [t], [t], [t], None, seed=0, **hyper)
    with pytest.raises(TypeError, match="CUDA tensor"):
        mqg.mqg_layer_norm(t, 1, 8, None, None, 1e-5, t)
    with pytest.raises(TypeError, match="CUDA tensor"):
        mqg.mqg_layer_norm_grad(t, t, 1, 8, None, t, t, None, None, None)


BESIDE_CODEC = ["mqg_adamw.cu", "mqg_layer_norm.cu", "mqg_layer_norm_grad.cu"]


@pytest.mark.parametrize("name", BESIDE_CODEC)
def test_every_kernel_waits_for_the_launch_before_it(name):
    """Before it touches memory, under no condition: see the programmatic dependent launches of the other kernels."""
    source = (CSRC / name).read_text()
    bodies = dict(_bodies(source))
    assert len(bodies) == source.count("__global__") > 0
    for kernel, body in bodies.items():
        wait = re.search(r"^    grid_dependency_wait\(\);", body, re.M)
        assert wait, kernel
        assert not re.search(r"__ld\w+\(|atomic\w+\(|\.load\(|\.store\(|\bmemcpy|\bload\(|weight_at\(", body[:wait.start()]), kernel
