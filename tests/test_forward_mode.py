"""A dual tensor of forward-mode differentiation is refused by the calls that have gradients: none of them carries a tangent along."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2002_02645_b200 import binding as fb


def calls(dev):
    x, w = torch.zeros(4, 64, device=dev).bfloat16(), torch.zeros(16, 64, device=dev).bfloat16()
    bias, r, norm = torch.zeros(16, device=dev), torch.zeros(4, 16, device=dev), torch.ones(64, device=dev)
    q, k = torch.zeros(4, 2, 64, device=dev).bfloat16(), torch.zeros(4, 1, 64, device=dev).bfloat16()
    rope, pos = torch.zeros(8, 64, device=dev), torch.zeros(4, dtype=torch.int32, device=dev)
    return [(fb.linear, (x, w, bias), dict(residual=r)), (fb.layer_norm, (x, norm, norm.clone()), {}),
            (fb.head_norm_rope, (q, k, norm, norm.clone(), rope, pos), {})]


def each_dual(dev):
    for call, args, kw in calls(dev):
        for i, t in enumerate(args):
            if t.is_floating_point():
                yield call, i, args, kw


def check(dev):
    for call, i, args, kw in each_dual(dev):
        with forward_ad.dual_level():
            dual = list(args)
            dual[i] = forward_ad.make_dual(args[i], torch.ones_like(args[i]))
            with pytest.raises(ValueError, match="forward-mode"):
                call(*dual, **kw)
    call, args, kw = calls(dev)[0]
    with forward_ad.dual_level(), pytest.raises(ValueError, match="forward-mode"):
        call(*args, residual=forward_ad.make_dual(kw["residual"], torch.ones_like(kw["residual"])))


def test_refused_in_a_transform_too():
    for call, i, args, kw in each_dual("cpu"):
        with pytest.raises(ValueError, match="forward-mode"):
            torch.func.jvp(lambda t: call(*args[:i], t, *args[i + 1:], **kw), (args[i],), (torch.ones_like(args[i]),))


def test_refused_before_any_device_is_needed():
    check("cpu")


@pytest.mark.gpu
def test_refused_on_the_device_and_nothing_else_is():
    check("cuda")
    with forward_ad.dual_level():                             # (tensors without a tangent)
        for call, args, kw in calls("cuda"):
            call(*args, **kw)
