"""Settings of cuts as the binding takes them (no GPU)."""
import pytest
import torch

import paper_2506_05632_amd as llc
from paper_2506_05632_amd import binding


class Rows:
    """What the binding asks of logits on a device."""
    is_cuda, dtype, shape, device = True, torch.float32, (2, 8), torch.device("cuda:0")

    def dim(self):
        return 2

    def stride(self, at):
        return (8, 1)[at]

    def data_ptr(self):
        return 0x1000


def _args(**settings):
    a = binding.SampleArgs()
    binding._cut_into(a, "llc_sample", Rows(), "logits", **{**dict(temp=1.0, top_k=0, top_p=1.0, min_p=0.0), **settings})
    return a


@pytest.mark.parametrize("top_k", [-(1 << 32) + 5, -(1 << 31) - 1, 1 << 31, (1 << 32) + 5, 2.5])
@pytest.mark.parametrize("temp", [1.0, 1])
def test_numbers_that_32_bits_do_not_hold_are_refused(top_k, temp):
    with pytest.raises(ValueError, match="top_k"):
        _args(top_k=top_k, temp=temp)


@pytest.mark.parametrize("top_k", [0, 1, 50, (1 << 31) - 1, -1, -(1 << 31)])
@pytest.mark.parametrize("temp", [1.0, 1])
def test_numbers_arrive_as_they_are(top_k, temp):
    # (the library refuses the negative ones)
    a = _args(top_k=top_k, temp=temp)
    assert (a.top_k, a.temp, a.top_p, a.min_p) == (top_k, 1.0, 1.0, 0.0)
    a.R, a.V, a.S, a.u, a.tokens, a.flags = 2, 8, 1, 0x2000, 0x3000, llc.FLAG_DRY_RUN
    assert llc.load().llc_sample(a) == (0 if top_k >= 0 else -8)
