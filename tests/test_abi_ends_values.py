"""Host-side checks of the calls at the vocabulary's two ends, beyond those of test_abi_ends.py (no GPU)."""
import ctypes

import pytest

import paper_2506_05632_amd as llc
from paper_2506_05632_amd import binding
from test_abi_ends import GRAD, SCORES, _filled


@pytest.mark.parametrize("temp,code", [(2.0 ** -126, 0), (2.0 ** -127, -3), (1e-40, -3), (1e-45, -3)])
def test_a_temperature_is_a_normal_number(temp, code):
    # (log2(e) / temp and 1 / temp leave fp32 below: what has p = 1 would be inf - inf from itself)
    lib = llc.load()
    for kind, want in ((0, code), (2, 0)):  # (log weights take none)
        assert lib.llc_token_logprobs(ctypes.byref(_filled(binding.TokenLogprobsArgs, SCORES, dict(flags=4, temp=temp, kind=kind)))) == want
        assert lib.llc_token_logprobs_grad(ctypes.byref(_filled(binding.TokenLogprobsGradArgs, GRAD, dict(flags=4, temp=temp, kind=kind)))) == want
