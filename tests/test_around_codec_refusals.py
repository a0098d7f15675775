"""Calls of the norm, clipping and embedding operators that are refused before anything reaches the device.  No GPU needed:
the C ABI checks its arguments on the host, the binding its tensors."""
import ctypes as C
import math

import pytest
import torch

import paper_1804_08066_b200 as mqg

OK, INVALID, ALIGN = mqg.MQG_OK, mqg.MQG_ERR_INVALID, mqg.MQG_ERR_ALIGN
P, ODD2, ODD4, ODD8 = 0x10000, 0x10002, 0x10004, 0x10008       # never dereferenced on the host


@pytest.fixture(scope="module")
def lib():
    return mqg.raw_library()


def _list(*tensors):
    n = len(tensors)
    return ((C.c_void_p * n)(*(t[0] for t in tensors)), (C.c_uint64 * n)(*(t[1] for t in tensors)),
            (C.c_int * n)(*(t[2] for t in tensors)), n)


GOOD = ((P, 100, 0), (P + 4096, 7, 1))
FLOATS = 1 << 20


def test_lists_are_checked(lib):
    calls = [lambda l: lib.mqg_grad_norm(*l, 1.0, P, P, FLOATS, None),
             lambda l: lib.mqg_clip_grad_norm(*l, 1.0, P, P, FLOATS, None),
             lambda l: lib.mqg_clip_flatten(*l, 1.0, P, 0, P, P, FLOATS, None),
             lambda l: lib.mqg_scale_grads(*l, P, None)]
    for call in calls:
        assert call(_list((None, 5, 0))) == INVALID and "tensor 0 is null" in mqg.mqg_last_error()
        assert call(_list(GOOD[0], (P, 5, 2))) == INVALID and "dtype" in mqg.mqg_last_error()
        assert call(_list(GOOD[0], (ODD2, 5, 0))) == ALIGN and "tensor 1" in mqg.mqg_last_error()
        assert call(_list((P + 1, 5, 1))) == ALIGN
        assert call(_list((P, 1 << 42, 0))) == INVALID
        assert call(_list(*[(P, 1 << 41, 0)] * 3)) == INVALID
        p, s, d, n = _list(*GOOD)
        assert call((p, s, d, -1)) == INVALID
        for missing in ((None, s, d, n), (p, None, d, n), (p, s, None, n)):
            assert call(missing) == INVALID


def test_norm_arguments_are_checked(lib):
    good = _list(*GOOD)
    need = mqg.mqg_norm_workspace_floats(2)
    for call in (lambda m, r, w, f: lib.mqg_grad_norm(*good, m, r, w, f, None),
                 lambda m, r, w, f: lib.mqg_clip_grad_norm(*good, m, r, w, f, None),
                 lambda m, r, w, f: lib.mqg_clip_flatten(*good, m, P, 0, r, w, f, None)):
        for max_norm in (-1.0, -math.inf, math.nan):
            assert call(max_norm, P, P, need) == INVALID and "max_norm" in mqg.mqg_last_error()
        assert call(1.0, None, P, need) == INVALID and call(1.0, P + 2, P, need) == ALIGN
        assert call(1.0, P, None, need) == INVALID and call(1.0, P, ODD4, need) == ALIGN
        assert call(1.0, P, P, need - 1) == INVALID and "mqg_norm_workspace_floats" in mqg.mqg_last_error()
    assert lib.mqg_clip_flatten(*good, 1.0, None, 0, P, P, need, None) == INVALID
    assert lib.mqg_clip_flatten(*good, 1.0, ODD2, 0, P, P, need, None) == ALIGN
    assert lib.mqg_clip_flatten(*good, 1.0, P, 3, P, P, need, None) == INVALID
    assert lib.mqg_scale_grads(*good, None, None) == INVALID and lib.mqg_scale_grads(*good, ODD2, None) == ALIGN


def test_apply_clipped_is_checked(lib):
    assert lib.mqg_apply_clipped(None, None, 0.1, None, 0, None) == OK
    assert lib.mqg_apply_clipped(None, P, 0.1, P, 8, None) == INVALID
    assert lib.mqg_apply_clipped(P, None, 0.1, P, 8, None) == INVALID
    assert lib.mqg_apply_clipped(P, P, 0.1, None, 8, None) == INVALID
    assert lib.mqg_apply_clipped(ODD8, P, 0.1, P, 8, None) == ALIGN
    assert lib.mqg_apply_clipped(P, ODD4, 0.1, P, 8, None) == ALIGN
    assert lib.mqg_apply_clipped(P, P, 0.1, ODD2, 8, None) == ALIGN


def test_tables_are_checked(lib):
    big = 1 << 31
    need = mqg.mqg_embedding_workspace_floats(10, 20, 8)

    def lookup(table=P, tt=0, rows=20, dim=8, ids=P, it=1, tokens=10, out=P, ot=0):
        return lib.mqg_embedding(table, tt, rows, dim, ids, it, tokens, 1.0, out, ot, None)

    def grad(table=P, tt=0, rows=20, dim=8, ids=P, it=1, tokens=10, out=P, ot=0, work=P, floats=need, add=0):
        return lib.mqg_embedding_grad(out, ot, ids, it, tokens, rows, dim, 1.0, table, tt, add, work, floats, None)

    for call in (lookup, grad):
        assert call(rows=big) == INVALID and call(tokens=big) == INVALID and call(dim=(1 << 22) + 1) == INVALID
        assert call(tt=2) == INVALID and call(ot=-1) == INVALID and call(it=2) == INVALID
        assert call(ids=None) == INVALID and call(table=None) == INVALID and call(out=None) == INVALID
        assert call(ids=ODD4) == ALIGN and call(ids=ODD2, it=0) == ALIGN
        assert call(table=ODD2) == ALIGN and call(table=P + 1, tt=1) == ALIGN
        assert call(out=ODD2) == ALIGN and call(out=P + 1, ot=1) == ALIGN
        assert call(tokens=10, dim=0, ids=None, table=None, out=None) == OK
    assert lookup(tokens=0, ids=None, table=None, out=None) == OK
    assert grad(tokens=0, ids=None, table=None, out=None, add=1) == OK
    assert grad(rows=0, table=None, out=None) == OK
    assert grad(floats=need - 1) == INVALID and "mqg_embedding_workspace_floats" in mqg.mqg_last_error()
    assert grad(work=None) == INVALID and grad(work=ODD8) == ALIGN


def test_workspace_sizes():
    assert mqg.mqg_norm_workspace_floats(0) == mqg.mqg_norm_workspace_floats(1) == mqg.mqg_norm_workspace_floats(1024)
    assert mqg.mqg_norm_workspace_floats(1025) == 2 * mqg.mqg_norm_workspace_floats(1)
    assert mqg.mqg_embedding_workspace_floats(0, 5, 5) == mqg.mqg_embedding_workspace_floats(5, 0, 5) == 0
    assert mqg.mqg_embedding_workspace_floats(1 << 40, 5, 5) == 0


def test_cpu_tensors_and_wrong_types_are_refused():
    x, i = torch.zeros(64), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: mqg.mqg_grad_norm([x], 1.0, x, x), lambda: mqg.mqg_clip_grad_norm([x], 1.0, x, x),
                 lambda: mqg.mqg_clip_flatten([x], 1.0, x, x, x), lambda: mqg.mqg_scale_grads([x], x),
                 lambda: mqg.mqg_apply_clipped(x, x, 0.1, x, 64), lambda: mqg.mqg_embedding(x, 8, 8, i, 4, 1.0, x),
                 lambda: mqg.mqg_embedding_grad(x, i, 4, 8, 8, 1.0, x, x)):
        with pytest.raises(TypeError, match="CUDA tensor"):
            call()
    with pytest.raises(TypeError):
        mqg.mqg_grad_norm([x], 1.0, x)
    with pytest.raises(TypeError):
        mqg.mqg_embedding(x, 8, 8, i, 4, 1.0, x, padding=0)


@pytest.mark.skipif(torch.cuda.is_available(), reason="tells a launch by its error, which there is without a device only")
@pytest.mark.parametrize("count", [0, 2, 32, 33, 1024, 1025, 1500])
def test_lists_without_elements_are_launched(lib, count):
    """The result of a list of empty tensors is written by a launch like any other's: no call returns without one."""
    empty = _list(*[(None, 0, j % 2) for j in range(count)])
    need = mqg.mqg_norm_workspace_floats(count)
    assert lib.mqg_grad_norm(*empty, 1.0, P, P + 4096, need, None) == mqg.MQG_ERR_CUDA
    assert lib.mqg_clip_grad_norm(*empty, 1.0, P, P + 4096, need, None) == mqg.MQG_ERR_CUDA
    assert lib.mqg_clip_flatten(*empty, 1.0, None, 0, P, P + 4096, need, None) == mqg.MQG_ERR_CUDA


@pytest.mark.gpu
def test_sizes_types_and_overlaps_of_device_tensors():
    x, i = torch.zeros(64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    work, half = torch.zeros(FLOATS, device="cuda"), torch.zeros(64, dtype=torch.float16, device="cuda")
    res = torch.zeros(2, device="cuda")
    for error, match, call in (
            (ValueError, "result holds 1", lambda: mqg.mqg_grad_norm([x], 1.0, res[1:], work)),
            (TypeError, "result must be float32", lambda: mqg.mqg_grad_norm([x], 1.0, half, work)),
            (TypeError, "grads must be float32 or bfloat16", lambda: mqg.mqg_grad_norm([half], 1.0, res, work)),
            (ValueError, "contiguous", lambda: mqg.mqg_grad_norm([x[::2]], 1.0, res, work)),
            (ValueError, "flat holds 64", lambda: mqg.mqg_clip_flatten([x, x], 1.0, x.clone(), res, work)),
            (ValueError, r"grads\[1\] and flat share", lambda: mqg.mqg_clip_flatten([x.clone()[:8], x[11:]], 1.0, x, res, work)),
            (ValueError, r"grads\[0\] and grads\[2\] share", lambda: mqg.mqg_clip_grad_norm([x, x.clone(), x], 1.0, res, work)),
            (ValueError, r"grads\[0\] and grads\[1\] share", lambda: mqg.mqg_scale_grads([x[8:], x[:9]], res)),
            (ValueError, "params holds", lambda: mqg.mqg_apply_clipped(x, x.clone(), 0.1, res, 65)),
            (ValueError, "acc holds", lambda: mqg.mqg_apply_clipped(x, x[:60], 0.1, res, 64)),
            (ValueError, "table holds", lambda: mqg.mqg_embedding(x, 9, 8, i, 4, 1.0, x)),
            (ValueError, "table holds", lambda: mqg.mqg_embedding(x, 1 << 40, 1 << 40, i, 4, 1.0, x)),
            (ValueError, "ids holds", lambda: mqg.mqg_embedding(x, 8, 8, i, 5, 1.0, x)),
            (TypeError, "ids must be", lambda: mqg.mqg_embedding(x, 8, 8, x, 4, 1.0, x)),
            (ValueError, "out holds", lambda: mqg.mqg_embedding(x, 8, 8, i, 4, 1.0, x[:31])),
            (ValueError, "grad holds", lambda: mqg.mqg_embedding_grad(x, i, 4, 9, 8, 1.0, x, work)),
            (ValueError, "dout holds", lambda: mqg.mqg_embedding_grad(x, i, 4, 2, 17, 1.0, x, work)),
            (mqg.MqgError, "workspace holds 1", lambda: mqg.mqg_embedding_grad(x, i, 4, 8, 8, 1.0, x.clone(), work[:1]))):
        with pytest.raises(error, match=match):
            call()
    # neighbours that touch do not overlap, in any order
    mqg.mqg_scale_grads([x[32:], x[:32]], res + 1)
    assert mqg.mqg_device_timeouts() == 0
