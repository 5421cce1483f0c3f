"""What the calls on models of many classes refuse, and the sizes they ask for (no GPU needed: a refused call enqueues nothing)."""
import ctypes as C

import pytest

import paper_1805_10111_amd as dq
from paper_1805_10111_amd import api

F32, F16, BF16 = 0, 1, 2
AT = 1 << 20                                    # some address: never read


def problem(type=BF16, n=10, c=100, d=64, a=AT, lda=64, w=AT, ldw=64):
    return api._Classes(type, n, c, d, a, lda, w, ldw)


def teacher(k=4, cls=AT, logit=AT, ld=4, tau=1.0):
    return api._Teacher(k, cls, logit, ld, tau)


def size(p, op=dq.OP_CLASS_GRAD, k=0):
    return api._lib.dq_class_workspace_bytes(op, C.byref(p), k)


def loss(p, label=AT, out=AT, ws=AT, nbytes=1 << 40):
    return api._lib.dq_class_loss(C.byref(p), label, out, None, None, ws, nbytes, None)


def distill(p, t, out=AT, ws=AT, nbytes=1 << 40):
    return api._lib.dq_distill_loss(C.byref(p), C.byref(t), out, None, None, ws, nbytes, None)


def grad(p, da=AT, ldda=64, dw=AT, lddw=64, ws=AT, nbytes=1 << 40):
    return api._lib.dq_class_grad(C.byref(p), AT, None, 1.0, None, None, da, ldda, dw, lddw, None, ws, nbytes, None)


BAD = [dict(type=3), dict(type=-1), dict(n=0), dict(c=0), dict(d=0), dict(n=-5), dict(a=None), dict(w=None), dict(lda=63), dict(ldw=1),
       dict(a=AT + 1), dict(type=F32, w=AT + 2)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_problems(bad):
    p = problem(**bad)
    assert size(p) == loss(p) == grad(p) == distill(p, teacher()) == dq.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(d=(1 << 20) + 1, lda=1 << 22, ldw=1 << 22), dict(lda=(1 << 22) + 1), dict(c=(1 << 30) + 1),
                                 dict(n=(1 << 30) + 1)], ids=str)
def test_problems_that_are_too_large(bad):
    p = problem(**bad)
    assert size(p) == loss(p) == dq.ERR_UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(k=0), dict(k=-1), dict(cls=None), dict(logit=None), dict(ld=3), dict(tau=0.0), dict(tau=-1.0),
                                 dict(tau=float("nan")), dict(tau=float("inf"))], ids=str)
def test_teachers(bad):
    assert distill(problem(), teacher(**bad)) == dq.ERR_INVALID_ARG


def test_teachers_that_are_too_wide():
    assert distill(problem(), teacher(k=1025, ld=1025)) == dq.ERR_UNSUPPORTED
    assert size(problem(), k=1025) == dq.ERR_UNSUPPORTED and size(problem(), k=-1) == dq.ERR_INVALID_ARG


def test_other_arguments():
    p = problem()
    assert size(p, op=1) == dq.ERR_INVALID_ARG
    assert loss(p, label=None) == loss(p, out=None) == loss(p, ws=None) == loss(p, ws=AT + 8) == dq.ERR_INVALID_ARG
    assert grad(p, ldda=63) == grad(p, lddw=1) == grad(p, da=AT + 1) == grad(p, dw=AT + 1) == dq.ERR_INVALID_ARG
    assert api._lib.dq_class_loss(None, AT, AT, None, None, AT, 1 << 40, None) == dq.ERR_INVALID_ARG
    assert api._lib.dq_distill_loss(C.byref(p), None, AT, None, None, AT, 1 << 40, None) == dq.ERR_INVALID_ARG


def test_workspaces_that_are_too_small():
    p = problem()
    small, large = size(p, dq.OP_CLASS_LOSS), size(p)
    assert 0 < small < large and small % 16 == large % 16 == 0
    assert loss(p, nbytes=small - 1) == grad(p, nbytes=large - 1) == dq.ERR_WORKSPACE


@pytest.mark.parametrize("t", [F32, BF16])
def test_the_workspace_does_not_hold_the_scores(t):
    """8192 rows over a million classes: pieces of 512 MB, the packed model where it is not read in place."""
    n, c, d = 8192, 1 << 20, 256
    p = problem(t, n, c, d, lda=d, ldw=d)
    model = 6 * c * d if t == F32 else 0
    sums = 12 * n * (c // 128)
    assert size(p) < (512 << 20) + model + sums + (1 << 30)
    assert size(p) < n * c * 2


def test_python_refuses_what_does_not_fit():
    import torch
    a = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        dq.DeviceClasses(a, a)                                  # not on the GPU
    with pytest.raises(TypeError):
        dq.DeviceClasses(a.double(), a.double())
    with pytest.raises(TypeError):
        dq.DeviceClasses(a, a.half())


# ------------------------------------------------------------------------------------------------ 4 bits
def mx4(n=10, d=200, codes=AT, ld_codes=128, scales=AT, ld_scales=8):
    return api._Mx4(n, d, codes, ld_codes, scales, ld_scales)


def scores(w, n=3, lda=200, ld=10, a=AT, out=AT, t=BF16, out_t=F32, ws=AT, nbytes=1 << 40):
    return api._lib.dq_mx4_scores(a, t, n, lda, C.byref(w), out, out_t, ld, None, ws, nbytes, None)


BAD4 = [dict(n=0), dict(d=0), dict(codes=None), dict(scales=None), dict(codes=AT + 8), dict(scales=AT + 2), dict(ld_codes=127), dict(ld_codes=64),
        dict(ld_codes=136), dict(ld_scales=4), dict(ld_scales=10), dict(d=300)]


@pytest.mark.parametrize("bad", BAD4, ids=str)
def test_matrices_in_four_bits(bad):
    q, good = mx4(**bad), mx4()
    lib = api._lib
    assert lib.dq_mx4_quantize(AT, F32, 1000, C.byref(q), None, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_dequantize(C.byref(q), AT, F32, 1000, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_product(C.byref(q), C.byref(good), AT, F32, 100, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_product(C.byref(good), C.byref(q), AT, F32, 100, None) == dq.ERR_INVALID_ARG
    assert scores(q) == dq.ERR_INVALID_ARG


def test_other_arguments_in_four_bits():
    q, lib = mx4(), api._lib
    assert lib.dq_mx4_quantize(None, F32, 200, C.byref(q), None, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_quantize(AT, 7, 200, C.byref(q), None, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_quantize(AT, F32, 199, C.byref(q), None, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_quantize(AT + 2, F32, 200, C.byref(q), None, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_dequantize(C.byref(q), AT + 1, F16, 200, None) == dq.ERR_INVALID_ARG
    other = mx4(d=130)
    assert lib.dq_mx4_product(C.byref(q), C.byref(other), AT, F32, 100, None) == dq.ERR_INVALID_ARG
    assert lib.dq_mx4_product(C.byref(q), C.byref(q), AT, F32, 9, None) == dq.ERR_INVALID_ARG
    assert scores(q, n=0) == scores(q, lda=199) == scores(q, ld=9) == scores(q, a=None) == scores(q, out=None) == dq.ERR_INVALID_ARG
    assert scores(q, t=3) == scores(q, out_t=-1) == scores(q, ws=None) == scores(q, ws=AT + 4) == dq.ERR_INVALID_ARG
    need = lib.dq_mx4_scores_bytes(3, 200)
    assert need >= 3 * (128 + 8) and need % 16 == 0 and scores(q, nbytes=need - 1) == dq.ERR_WORKSPACE
    assert lib.dq_mx4_scores_bytes(0, 5) == lib.dq_mx4_row_bytes(0) == lib.dq_mx4_row_scales(-1) == dq.ERR_INVALID_ARG
    assert scores(mx4(d=(1 << 23) + 1, ld_codes=1 << 23, ld_scales=1 << 20), lda=1 << 24) == dq.ERR_UNSUPPORTED
    assert dq.dq_mx4_row_bytes(129) == 128 and dq.dq_mx4_row_scales(129) == 8


@pytest.mark.parametrize("tau", [1e-39, 1e-45])
def test_temperatures_without_an_inverse(tau):
    assert distill(problem(), teacher(tau=tau)) == dq.ERR_INVALID_ARG
    assert distill(problem(), teacher(tau=1e-38), nbytes=0) == dq.ERR_WORKSPACE


@pytest.mark.parametrize("bad", [dict(n=1 << 20, c=1 << 19, d=8), dict(n=1 << 20, c=1 << 20, d=8), dict(n=1, c=1 << 30, d=8), dict(n=20, c=1 << 30, d=8),
                                 dict(n=1 << 28, c=2, d=8), dict(n=1 << 30, c=1 << 30, d=8)], ids=str)
@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_problems_that_no_launch_takes(t, bad):
    """A launch has fewer than 2^32 threads: 2^23 tiles of 512, 2^24 of 256, 2^28 rows of 16."""
    p = problem(t, **bad)
    assert size(p, dq.OP_CLASS_LOSS) == size(p, dq.OP_CLASS_GRAD) == loss(p) == grad(p) == dq.ERR_UNSUPPORTED


@pytest.mark.parametrize("good", [dict(n=1 << 20, c=(1 << 19) - 256, d=8), dict(n=1, c=(1 << 30) - 64, d=8), dict(n=20, c=(1 << 30) - 64, d=8),
                                  dict(n=(1 << 28) - 16, c=2, d=8)], ids=str)
def test_the_largest_problems_that_a_launch_takes(good):
    p = problem(BF16, **good)
    assert size(p, dq.OP_CLASS_LOSS) > 0 and size(p) > 0 and loss(p, nbytes=0) == dq.ERR_WORKSPACE


def test_teachers_of_more_rows_than_a_launch_takes():
    """One block of 64 threads a row: 2^26 rows."""
    few, many = problem(n=(1 << 26) - 1, c=2, d=8), problem(n=1 << 26, c=2, d=8)
    assert size(few, k=4) > 0 and distill(few, teacher(), nbytes=0) == dq.ERR_WORKSPACE
    assert size(many, k=4) == distill(many, teacher()) == dq.ERR_UNSUPPORTED and size(many) > 0


@pytest.mark.parametrize("n", [1, 16, 17, 64])
def test_products_in_four_bits_that_no_launch_takes(n):
    """2^24 tiles of 64 classes; refused before the rows are quantized."""
    w, a = mx4(n=1 << 30, d=128, ld_codes=64, ld_scales=4), mx4(n=n, d=128, ld_codes=64, ld_scales=4)
    assert api._lib.dq_mx4_product(C.byref(a), C.byref(w), AT, BF16, 1 << 30, None) == dq.ERR_UNSUPPORTED
    assert scores(w, n=n, ld=1 << 30) == dq.ERR_UNSUPPORTED


@pytest.mark.parametrize("t,planes,wide", [(F32, 3, 256), (F16, 1, 256), (BF16, 1, 256)])
def test_the_workspace_holds_one_piece_of_gradients(t, planes, wide):
    """8192 rows of a million classes: 1 GB of g, three sums a tile and row, packed operands; and what is small beside these (da's partial sums,
    one value a row: below 128 MB)."""
    n, c, d = 8192, 1 << 20, 256
    known = 12 * n * (c // wide) + 2 * planes * n * d + (2 * planes * (n + c) * d if t == F32 else 0)
    piece = size(problem(t, n, c, d, lda=d, ldw=d)) - known
    assert (1 << 30) - 2 * planes * n * 256 <= piece <= (1 << 30) + (128 << 20)
