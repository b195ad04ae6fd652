"""Clipping where the norm leaves its type (needs an MI355X)."""
import math

import pytest
import torch

import paper_2506_05632_amd as llc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n", [1, 3, 1500])  # (joined by the second pass, and by a launch of its own)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_norm_beyond_its_type_leaves_the_gradients(n, dtype):
    grads = [torch.full((4 if n < 100 else 9000,), 3e38, device=DEV).to(dtype) for _ in range(n)]
    mine, out = [t.clone() for t in grads], [torch.zeros_like(t) for t in grads]
    for most in (1e-3, 1.0, 3e38, math.inf):
        assert llc.llc_clip_grad_norm(mine, most)["norm"].item() == math.inf
        assert llc.llc_clip_grad_norm(grads, most, out=out)["norm"].item() == math.inf
        assert all(torch.equal(u, v) and torch.equal(u, w) for u, v, w in zip(grads, mine, out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_norm_just_inside_its_type_scales_them(dtype):
    grads = [torch.full((4,), 1.5e38, device=DEV).to(dtype)]
    want = grads[0].double() / (2.0 * grads[0][0].double())
    found = llc.llc_clip_grad_norm(grads, 1.0)["norm"]
    assert torch.isfinite(found)
    # (the factor, some 2^-128, is a subnormal fp32 number: 2^-149 of it at most is lost)
    assert ((grads[0].double() - want).abs() <= 2.0 ** -8 * want + 2.0 ** -150 * 1.6e38).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [0.01, 0.7, 1.0 / 3.0, 1.9e-5, 0.63275796])
@pytest.mark.parametrize("n", [7, 8192, 28672, 1000003])
def test_the_norm_of_equal_entries_is_rounded_once(n, value, dtype):
    # equal squares round alike wherever they are added up, so that what sums lose does not average out
    grads = [torch.full((n,), value, device=DEV).to(dtype) for _ in range(3)]
    want = math.sqrt(3 * n) * grads[0][0].item()
    found = llc.llc_clip_grad_norm(grads, math.inf)["norm"].item()
    assert abs(found - want) <= 2.0 ** -24 * want * (1.0 + 2.0 ** -20)
