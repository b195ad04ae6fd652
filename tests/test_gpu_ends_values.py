"""Values that rows of logits may hold, beyond those of test_gpu_ends_scores.py: NaN of either kind among numbers, large finite
masks, long rows of equal entries (needs an MI355X).  Tolerances are ends_util's."""
import numpy as np
import pytest
import torch

import ends_util as ref
import paper_2506_05632_amd as llc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
SIGNALLING = {F32: (torch.int32, 0x7F800001), BF16: (torch.int16, 0x7F81)}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(R, V, dtype, seed, scale=2.0):
    return (scale * torch.randn(R, V, generator=_gen(seed), device=DEV)).to(dtype)


def _signal(x, row, columns, negative=False):
    """NaNs of the signalling kind, put in as bits: as a value they would be quieted."""
    whole, bits = SIGNALLING[x.dtype]
    x.view(whole)[row, columns] = bits - (1 << (8 * x.element_size() - 1)) if negative else bits


def _with_signalling(V, dtype):
    """Rows whose NaNs of the signalling kind lie beside, before and behind what counts."""
    x = _rows(20, V, dtype, V)
    everywhere = torch.arange(V, device=DEV)
    for r in range(16):  # the row's largest entry at every place of a lane's loads, a NaN on either side of it
        at = (37 * r) % (V - 2) + 1
        x[r, at] = 9.0 + 0.5 * r
        _signal(x, r, [at - 1, at + 1] if r % 3 == 0 else [at + 1] if r % 3 == 1 else [at - 1], r % 2 == 1)
    x[16] = torch.linspace(-6, 6, V, device=DEV).to(dtype)  # (offers every entry to the lists)
    _signal(x, 16, everywhere[everywhere % 3 == 1])
    x[17, 1::4] = float("inf")
    _signal(x, 17, everywhere[everywhere % 4 == 2])
    _signal(x, 18, everywhere)
    x[18, V // 2] = -1.0
    _signal(x, 19, everywhere, True)
    return x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [61, 1030, 9001, 40003, 70001])
def test_scores_beside_signalling_NaNs(V, dtype):
    x = _with_signalling(V, dtype)
    t = torch.randint(0, V, (20, 5), generator=_gen(V), device=DEV).to(torch.int32)
    t[:, 0] = (torch.arange(20, device=DEV) * 37) % (V - 2) + 1
    for M in (1, 20, 128):
        for chunks in (0, 1, 3):
            ref.check_scores(llc.llc_token_logprobs(x, t, M, temp=0.8, want_lse=True, v_chunks=chunks), x, t, M, 0.8)
