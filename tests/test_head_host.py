"""Refusals of the head's operators that need no GPU: the library's own checks of sizes, types, pointers and
alignment, and the binding's checks of tensors."""
import ctypes as C
import os

import pytest
import torch

from paper_1412_1576_amd import lda

OUT = 1 << 21


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lda.LIB_PATH):
        from paper_1412_1576_amd import build
        build.build_library()
    return lda.load_library()


def message(lib):
    return lib.lda_last_error(None).decode()


def norm(**kw):
    r = lda.lda_norm_rows()
    r.rows, r.width, r.x, r.x_stride, r.eps = 4, 100, 1 << 20, 100, 1e-6
    r.residual, r.residual_stride, r.weight = 1 << 20, 100, 1 << 20
    r.x_type = r.sum_type = r.weight_type = 2
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def gradients(**kw):
    g = lda.lda_norm_gradients()
    g.y_grad = g.sum_grad = g.sum = g.stats = 1 << 20
    g.y_grad_stride = g.sum_grad_stride = g.sum_stride = 100
    g.x_grad = g.residual_grad = g.weight_grad = g.workspace = OUT
    g.x_grad_stride = g.residual_grad_stride = 100
    g.workspace_bytes = 1 << 20
    for k, v in kw.items():
        setattr(g, k, v)
    return g


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(width=0), dict(x_type=3), dict(weight_type=-1), dict(sum_type=4), dict(sum_type=1),
    dict(weight_type=1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(weight=(1 << 20) + 1),
    dict(x=None), dict(x=(1 << 20) + 1), dict(residual=(1 << 20) + 1), dict(reserved_word=1)])
def test_norm_refuses(lib, kw):
    r = norm(**kw)
    assert lib.lda_norm(r, OUT, 100, OUT, 100, OUT) == lda.LDA_ERR_ARG and "lda_norm:" in message(lib)
    assert lib.lda_norm_bytes(r, 0, OUT, 100, OUT, OUT, 100) == lda.LDA_ERR_ARG and "lda_norm_bytes:" in message(lib)
    if not set(kw) & {"x", "residual"}:  # the gradient looks at the sum instead
        assert lib.lda_norm_grad(r, gradients()) == lda.LDA_ERR_ARG
        assert lib.lda_norm_grad_workspace(r) == lda.LDA_ERR_ARG


def test_rows_that_are_too_long(lib):
    assert lib.lda_norm(norm(width=(1 << 30) + 1, rows=1), OUT, 1 << 31, OUT, 1 << 31, OUT) == lda.LDA_ERR_UNSUPPORTED
    assert lib.lda_norm_grad_workspace(norm(width=(1 << 30) + 1)) == lda.LDA_ERR_UNSUPPORTED
    assert lib.lda_product_workspace(product(rows=1 << 31, classes=513)) == lda.LDA_ERR_UNSUPPORTED
    assert "2^40" in message(lib)


def test_norm_refuses_outputs(lib):
    r = norm()
    for args in ((None, 100, OUT, 100, OUT), (OUT + 1, 100, OUT, 100, OUT), (OUT, 99, OUT, 100, OUT),
                 (OUT, 100, None, 100, OUT), (OUT, 100, OUT + 1, 100, OUT), (OUT, 100, OUT, 99, OUT),
                 (OUT, 100, OUT, 100, OUT + 4)):
        assert lib.lda_norm(r, *args) == lda.LDA_ERR_ARG, args
    for args in ((2, OUT, 100, OUT, OUT, 100), (-1, OUT, 100, OUT, OUT, 100), (0, None, 100, OUT, OUT, 100),
                 (0, OUT, 100, None, OUT, 100), (0, OUT, 100, OUT + 2, OUT, 100), (1, OUT, 99, OUT, OUT, 100),
                 (1, OUT, 100, OUT, None, 100)):
        assert lib.lda_norm_bytes(r, *args) == lda.LDA_ERR_ARG, args
    assert lib.lda_norm(None, OUT, 100, OUT, 100, OUT) == lda.LDA_ERR_ARG
    r.reserved[3] = 1
    assert lib.lda_norm(r, OUT, 100, OUT, 100, OUT) == lda.LDA_ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(y_grad=None), dict(sum=None), dict(stats=None), dict(y_grad=(1 << 20) + 1), dict(sum_grad=(1 << 20) + 1),
    dict(stats=(1 << 20) + 4), dict(x_grad=OUT + 1), dict(residual_grad=OUT + 1), dict(weight_grad=OUT + 1),
    dict(x_grad_stride=99), dict(residual_grad_stride=99), dict(workspace=None), dict(workspace_bytes=4 * 400 - 1),
    dict(workspace=OUT + 8)])
def test_norm_gradient_refuses(lib, kw):
    assert lib.lda_norm_grad_workspace(norm()) == 4 * 400
    assert lib.lda_norm_grad(norm(), gradients(**kw)) == lda.LDA_ERR_ARG and "lda_norm_grad:" in message(lib)


def test_norm_of_no_rows(lib):
    r = norm(rows=0, x=None)
    assert lib.lda_norm(r, None, 0, None, 0, None) == lda.LDA_OK
    assert lib.lda_norm_bytes(r, 0, None, 0, None, None, 0) == lda.LDA_OK
    assert lib.lda_norm_grad_workspace(r) == 0
    assert lib.lda_norm_grad(r, gradients(weight_grad=None)) == lda.LDA_OK
    assert lib.lda_norm_grad(r, None) == lda.LDA_ERR_ARG
    g = gradients(weight_grad=None)
    g.reserved[0] = 1
    assert lib.lda_norm_grad(r, g) == lda.LDA_ERR_ARG


def test_struct_layouts():
    assert C.sizeof(lda.lda_norm_rows) == 8 + 8 + 2 * 16 + 8 + 4 * 4 + 8 + 16
    assert C.sizeof(lda.lda_norm_gradients) == 3 * 16 + 8 + 2 * 16 + 8 + 16 + 16


def test_the_binding_refuses_host_tensors():
    from paper_1412_1576_amd import operators
    for call in (operators.rms_norm, operators.rms_norm_8bit):
        with pytest.raises(ValueError, match="on the GPU"):
            call(torch.zeros(2, 5))
        with pytest.raises(ValueError, match="on the GPU"):
            call(None)


def log_probs(**kw):
    r = lda.lda_log_prob_rows()
    r.rows, r.classes, r.top, r.logits, r.logits_stride = 4, 1000, 8, 1 << 20, 1000
    r.tokens, r.tokens_stride, r.temperature = 1 << 20, 1, 1.0
    for k, v in kw.items():
        setattr(r, k, v)
    r.workspace, r.workspace_bytes = 1 << 20, 1 << 30
    return r


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, lda.LDA_ERR_ARG), ("classes", 0, lda.LDA_ERR_ARG), ("top", -1, lda.LDA_ERR_ARG),
    ("top", 257, lda.LDA_ERR_UNSUPPORTED), ("logits_type", 3, lda.LDA_ERR_ARG), ("tokens_type", 2, lda.LDA_ERR_ARG),
    ("temperature", 0.0, lda.LDA_ERR_ARG), ("temperature", float("nan"), lda.LDA_ERR_ARG),
    ("temperature", float("inf"), lda.LDA_ERR_ARG), ("temperature", 2.0 ** -11, lda.LDA_ERR_ARG),
    ("logits", None, lda.LDA_ERR_ARG), ("tokens", None, lda.LDA_ERR_ARG), ("logits", (1 << 20) + 2, lda.LDA_ERR_ARG),
    ("tokens", (1 << 20) + 2, lda.LDA_ERR_ARG), ("reserved_word", 1, lda.LDA_ERR_ARG)])
def test_log_probs_refuse(lib, field, value, code):
    r = log_probs(**{field: value})
    for call, args in (("lda_log_probs_workspace", ()), ("lda_log_probs", (OUT, OUT, OUT, OUT, OUT)),
                       ("lda_log_probs_grad", (OUT, OUT, 1, OUT, 1, OUT, 1000))):
        assert getattr(lib, call)(r, *args) == code, call
        assert call in message(lib)


def test_log_probs_refuse_outputs_and_workspaces(lib):
    r = log_probs()
    for args in ((None, OUT, OUT, OUT, OUT), (OUT, OUT, None, OUT, OUT), (OUT, OUT, OUT, None, OUT),
                 (OUT + 2, OUT, OUT, OUT, OUT), (OUT, OUT + 1, OUT, OUT, OUT), (OUT, OUT, OUT, OUT, OUT + 8)):
        assert lib.lda_log_probs(r, *args) == lda.LDA_ERR_ARG, args
    for args in ((None, OUT, 1, OUT, 1, OUT, 1000), (OUT, OUT, 1, OUT, 1, None, 1000), (OUT + 8, OUT, 1, OUT, 1, OUT, 1000),
                 (OUT, OUT + 2, 1, OUT, 1, OUT, 1000), (OUT, OUT, 1, OUT + 2, 1, OUT, 1000), (OUT, OUT, 1, OUT, 1, OUT + 2, 1000),
                 (OUT, OUT, 1, OUT, 1, OUT, 999)):
        assert lib.lda_log_probs_grad(r, *args) == lda.LDA_ERR_ARG, args
    big = log_probs(rows=1, classes=1_000_000, logits_stride=1_000_000)
    need = lib.lda_log_probs_workspace(big)
    assert need > 0
    for pointer, nbytes in ((None, need), (1 << 21, need - 1), ((1 << 21) + 8, need)):
        big.workspace, big.workspace_bytes = pointer, nbytes
        assert lib.lda_log_probs(big, OUT, OUT, OUT, OUT, OUT) == lda.LDA_ERR_ARG and "workspace" in message(lib)
    assert lib.lda_log_probs_workspace(None) == lda.LDA_ERR_ARG
    r.reserved[1] = 1
    assert lib.lda_log_probs(r, OUT, OUT, OUT, OUT, OUT) == lda.LDA_ERR_ARG
    none = log_probs(rows=0, logits=None, tokens=None)
    assert lib.lda_log_probs_workspace(none) == 0
    assert lib.lda_log_probs(none, None, None, None, None, None) == lda.LDA_OK
    assert lib.lda_log_probs_grad(none, None, None, 0, None, 0, None, 0) == lda.LDA_OK
    assert C.sizeof(lda.lda_log_prob_rows) == 8 + 8 + 2 * 16 + 8 + 8 + 24 + 16


def test_log_probs_binding_refuses_host_tensors():
    from paper_1412_1576_amd import operators
    with pytest.raises(ValueError, match="on the GPU"):
        operators.token_log_probs(torch.zeros(2, 5), torch.zeros(2, dtype=torch.int64))


def product(**kw):
    r = lda.lda_product_rows()
    r.rows, r.classes, r.width, r.out_type = 4, 1000, 64, 2
    r.a = r.b = r.a_scale = r.b_scale = 1 << 20
    r.a_stride = r.b_stride = 64
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, lda.LDA_ERR_ARG), ("classes", 0, lda.LDA_ERR_ARG), ("width", -1, lda.LDA_ERR_ARG),
    ("width", 131_072, lda.LDA_ERR_UNSUPPORTED), ("rows", (1 << 31) + 1, lda.LDA_ERR_UNSUPPORTED),
    ("out_type", 3, lda.LDA_ERR_ARG), ("a", None, lda.LDA_ERR_ARG), ("b", None, lda.LDA_ERR_ARG),
    ("a_scale", None, lda.LDA_ERR_ARG), ("b_scale", None, lda.LDA_ERR_ARG), ("a_scale", (1 << 20) + 2, lda.LDA_ERR_ARG),
    ("b_scale", (1 << 20) + 1, lda.LDA_ERR_ARG), ("reserved_word", 1, lda.LDA_ERR_ARG)])
def test_product_refuses(lib, field, value, code):
    r = product(**{field: value})
    assert lib.lda_product_workspace(r) == code and "lda_product_workspace" in message(lib)
    assert lib.lda_product(r, OUT, 1000) == code and "lda_product:" in message(lib)


def test_product_refuses_outputs_and_workspaces(lib):
    for args in ((None, 1000), (OUT + 1, 1000), (OUT, 999)):
        assert lib.lda_product(product(), *args) == lda.LDA_ERR_ARG
    assert lib.lda_product(None, OUT, 1000) == lda.LDA_ERR_ARG
    assert lib.lda_product_workspace(None) == lda.LDA_ERR_ARG
    r = product()
    r.reserved[0] = 1
    assert lib.lda_product(r, OUT, 1000) == lda.LDA_ERR_ARG
    r = product(rows=100, classes=100, width=16_384)
    need = lib.lda_product_workspace(r)
    assert need > 0
    for pointer, nbytes in ((None, need), (1 << 21, need - 1), ((1 << 21) + 8, need)):
        r.workspace, r.workspace_bytes = pointer, nbytes
        assert lib.lda_product(r, OUT, 1000) == lda.LDA_ERR_ARG and "workspace" in message(lib)
    none = product(rows=0, a=None, b=None, a_scale=None)
    assert lib.lda_product_workspace(none) == 0 and lib.lda_product(none, None, 0) == lda.LDA_OK
    assert C.sizeof(lda.lda_product_rows) == 8 + 8 + 16 + 8 + 16 + 8 + 8 + 24 + 16


def test_which_sides_of_a_product_are_packed(lib):
    """Above 128 rows, where a side does not lie in pieces of 16 bytes less than 2^22 apart; both where the width is no
    multiple of 16."""
    def need(rows, width=1008, **kw):
        return lib.lda_product_workspace(product(rows=rows, classes=200_000, width=width, **{"a_stride": 1008, "b_stride": 1008, **kw}))
    assert need(128, width=1000) == need(128, b_stride=1009) == need(129) == 0
    assert need(129, width=1000) == (129 + 200_000) * 1008
    assert need(129, a=(1 << 20) + 1) == need(129, a_stride=1 << 22) == need(129, a_stride=1009) == 129 * 1008
    assert need(129, b=(1 << 20) + 8) == need(129, b_stride=1024 + 8) == 200_000 * 1008


def test_product_binding_refuses_host_tensors():
    from paper_1412_1576_amd import operators
    x = torch.zeros(2, 8, dtype=torch.int8)
    with pytest.raises(ValueError, match="on the GPU"):
        operators.int8_matmul(x, torch.ones(2), x, torch.ones(2))


def test_a_derivative_is_wanted():
    """By leaves where gradients are on, by tangents of forward mode everywhere."""
    from torch.autograd import forward_ad

    from paper_1412_1576_amd import operators
    x = torch.ones(2, 5)
    leaf = x.clone().requires_grad_(True)
    assert not operators._wants_gradient(x, None) and operators._wants_gradient(None, x, leaf)
    with torch.no_grad():
        assert not operators._wants_gradient(leaf)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, x)
        assert operators._wants_gradient(None, x, dual) and not operators._wants_gradient(x, None, "x")
        with torch.no_grad():
            assert operators._wants_gradient(dual) and not operators._wants_gradient(leaf, dual.detach())
