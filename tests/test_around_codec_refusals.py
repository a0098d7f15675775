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


A, B, C_, D = 0x100000, 0x200000, 0x300000, 0x4000000       # apart from each other


def _refused(status, *names):
    return status == INVALID and "share memory" in mqg.mqg_last_error() and all(n in mqg.mqg_last_error() for n in names)


@pytest.mark.parametrize("form", ["norm", "in place", "flatten"])
def test_what_the_norm_writes_lies_apart(lib, form):
    need = mqg.mqg_norm_workspace_floats(2)

    def call(result=B, work=C_, flat=D, tensors=((A, 100, 0), (A + 400, 8, 1)), floats=need):
        l = _list(*tensors)
        if form == "norm":
            return lib.mqg_grad_norm(*l, 1.0, result, work, floats, None)
        if form == "in place":
            return lib.mqg_clip_grad_norm(*l, 1.0, result, work, floats, None)
        return lib.mqg_clip_flatten(*l, 1.0, flat, 1, result, work, floats, None)

    assert _refused(call(result=A + 396), "tensor 0", "result") and _refused(call(result=A), "tensor 0", "result")
    assert _refused(call(result=A + 412), "tensor 1", "result") and _refused(call(result=A - 4), "tensor 0", "result")
    assert _refused(call(work=A + 408), "tensor 1", "workspace")
    assert _refused(call(work=A - 4 * need + 8), "tensor 0", "workspace")
    assert _refused(call(result=C_), "result", "workspace") and _refused(call(result=C_ - 4), "result", "workspace")
    assert _refused(call(result=C_ + 4 * need - 4), "result", "workspace")
    # what is behind the floats that a call needs is not touched, nor are empty tensors
    others = [dict(result=A - 8), dict(result=A + 416), dict(work=A + 416), dict(work=A - 4 * need),
              dict(result=C_ + 4 * need, floats=need + 8), dict(tensors=((B, 0, 0), (A, 8, 0)))]
    if form == "flatten":
        assert _refused(call(flat=A + 414), "tensor 1", "flat") and _refused(call(flat=A - 214), "tensor 0", "flat")
        assert _refused(call(flat=B - 214), "flat", "result") and _refused(call(flat=C_ + 4 * need - 2), "flat", "workspace")
        others += [dict(flat=A + 416), dict(flat=A - 216), dict(flat=B - 216), dict(flat=C_ + 4 * need)]
    if not torch.cuda.is_available():                   # (what is not refused fails at the launch here)
        assert all(call(**o) == mqg.MQG_ERR_CUDA for o in others)


def test_a_factor_lies_apart(lib):
    l = _list((A, 100, 0), (A + 400, 8, 1))
    assert _refused(lib.mqg_scale_grads(*l, A + 396, None), "tensor 0", "factor")
    assert _refused(lib.mqg_scale_grads(*l, A + 412, None), "tensor 1", "factor")
    assert _refused(lib.mqg_apply_clipped(A, B, 0.1, A + 396, 100, None), "params", "factor")
    assert _refused(lib.mqg_apply_clipped(A, A + 384, 0.1, B, 100, None), "params", "acc")
    assert _refused(lib.mqg_apply_clipped(A, A - 384, 0.1, B, 100, None), "params", "acc")
    if not torch.cuda.is_available():
        assert lib.mqg_scale_grads(*l, A + 416, None) == lib.mqg_scale_grads(*l, A - 4, None) == mqg.MQG_ERR_CUDA
        assert lib.mqg_apply_clipped(A, A + 400, 0.1, B, 100, None) == mqg.MQG_ERR_CUDA
        assert lib.mqg_apply_clipped(A, A, 0.1, A + 400, 100, None) == mqg.MQG_ERR_CUDA      # element by element: in place


def test_tables_and_rows_lie_apart(lib):
    need = mqg.mqg_embedding_workspace_floats(10, 20, 8)

    def lookup(table=A, ids=B, out=C_, it=1):           # 20 rows of 32 bytes, 10 ids, 10 rows of 16 bytes
        return lib.mqg_embedding(table, 0, 20, 8, ids, it, 10, 1.0, out, 1, None)

    def grad(dout=A, ids=B, table=C_, work=D, tokens=10, floats=need):      # 10 rows of 32 bytes, 10 ids, 20 rows of 16 bytes
        return lib.mqg_embedding_grad(dout, 0, ids, 1, tokens, 20, 8, 1.0, table, 1, 0, work, floats, None)

    assert _refused(lookup(out=A), "out", "table") and _refused(lookup(out=A + 638), "out", "table")
    assert _refused(lookup(out=A - 158), "out", "table") and _refused(lookup(out=B), "out", "ids")
    assert _refused(lookup(out=B + 38, it=0), "out", "ids") and _refused(lookup(out=B + 78), "out", "ids")
    assert _refused(grad(table=A), "grad", "dout") and _refused(grad(table=A + 318), "grad", "dout")
    assert _refused(grad(table=B - 318), "grad", "ids") and _refused(grad(table=D + 4 * need - 2), "grad", "workspace")
    assert _refused(grad(work=A + 304), "workspace", "dout") and _refused(grad(work=B + 64), "workspace", "ids")
    if not torch.cuda.is_available():
        for status in (lookup(out=A + 640), lookup(out=A - 160), lookup(out=B + 40, it=0), lookup(out=B + 80), lookup(ids=A),
                       grad(table=A + 320), grad(table=B - 320), grad(table=D + 4 * need, floats=need + 8),
                       grad(work=A + 320), grad(work=B + 80), grad(ids=A), grad(dout=C_, tokens=0)):
            assert status == mqg.MQG_ERR_CUDA


def test_cluster_sizes_of_the_test_hook(lib):
    for most in (3, 12, 17, 32, 1 << 31):
        assert lib.mqg_test_sort_cluster(most) == INVALID
    for most in (16, 8, 4, 2, 1, 0):
        assert lib.mqg_test_sort_cluster(most) == OK


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


@pytest.mark.gpu
def test_device_tensors_that_share_memory():
    x, i = torch.zeros(4096, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    res, work, y = torch.zeros(2, device="cuda"), torch.zeros(FLOATS, device="cuda"), torch.zeros(64, device="cuda")
    for call in (lambda: mqg.mqg_grad_norm([y, x], 1.0, x[8:], work), lambda: mqg.mqg_clip_grad_norm([y, x], 1.0, res, x),
                 lambda: mqg.mqg_clip_flatten([y], 1.0, x, x[60:], work), lambda: mqg.mqg_scale_grads([y, x], x[4095:]),
                 lambda: mqg.mqg_apply_clipped(x, x[4:], 0.1, res, 64), lambda: mqg.mqg_embedding(x, 8, 4, i, 4, 1.0, x[31:]),
                 lambda: mqg.mqg_embedding_grad(x, i, 4, 8, 8, 1.0, x[31:], work),
                 lambda: mqg.mqg_embedding_grad(x, i, 4, 8, 8, 1.0, y, x)):
        with pytest.raises(mqg.MqgError, match="share memory"):
            call()
    mqg.mqg_embedding(x, 8, 4, i, 4, 1.0, x[32:])
    mqg.mqg_embedding_grad(x, i, 4, 8, 8, 1.0, x[32:], work)
    mqg.mqg_apply_clipped(x, x, 0.1, res, 64)
