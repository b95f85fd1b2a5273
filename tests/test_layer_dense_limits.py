"""Argument blocks that are refused before any device is needed: limits of waits, and the gradient of a float32 result."""
import pytest

from paper_2002_02645_b200 import binding as fb


def backward(**kw):
    a = fb.fi_linear_backward_t(x=1 << 20, weight=1 << 21, dy=1 << 22, dx=1 << 23, dweight=1 << 24, workspace=1 << 25, x_stride=64, weight_stride=64,
                                dy_stride=32, preact_stride=32, dx_stride=64, dweight_stride=64, tokens=4, in_dim=64, out_dim=32)
    for k, v in kw.items():
        setattr(a, k, v)
    return fb.load_library().fi_linear_backward(bytes(a), None)


@pytest.mark.parametrize("bad", [dict(wait_limit=-1), dict(dy_f32=1, workspace=None), dict(dy_f32=1, dy=(1 << 22) + 8), dict(dy_f32=1, dy_stride=34),
                                 dict(dy_f32=1, dy_stride=28), dict(dy_f32=1, dy=None), dict(dy_stride=28), dict(dy=(1 << 22) + 4)], ids=str)
def test_gradients_of_products(bad):
    assert backward(**bad) == fb.FI_ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["fi_layer_norm", "fi_layer_norm_backward"])
def test_norm(call):
    a = fb.fi_layer_norm_t(x=1 << 20, dy=1 << 21, out=1 << 22, x_stride=64, dy_stride=64, out_stride=64, tokens=4, dim=64, eps=1e-5, wait_limit=-1)
    assert getattr(fb.load_library(), call)(bytes(a), None) == fb.FI_ERR_INVALID_ARG


def test_a_result_of_no_rows_needs_no_place_but_what_is_read_has_to_be_there():
    lib = fb.load_library()
    a = fb.fi_linear_t(x=1 << 20, weight=1 << 21, rows=1 << 23, x_stride=64, weight_stride=64, out_stride=32, tokens=4, in_dim=64, out_dim=32)
    assert lib.fi_linear(bytes(a), None) == fb.FI_OK                  # nothing to do
    a.preact, a.preact_stride, a.x = 1 << 24, 32, None
    assert lib.fi_linear(bytes(a), None) == fb.FI_ERR_INVALID_ARG
