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


def _check_grad(x, t, a, b, temp, out, rows):
    """`rows` of a gradient, and of the scores beside it."""
    part = lambda v: None if v is None else v[rows]  # noqa: E731
    want, tol = ref.gradient(x[rows], t[rows], a[rows], part(b), temp)
    far = np.abs(out["grad"][rows].detach().cpu().double().numpy() - want) - tol
    assert far.max() <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))
    if "logp" in out:
        ref.check_scores({k: v[rows] for k, v in out.items()}, x[rows], t[rows], 0, temp)


def _gradients(x, t, a, b, temp, rows):
    """Every way to the gradient: in one pass (or over split rows), over rows split in three, in place, from given sums."""
    for chunks in (0, 3):
        _check_grad(x, t, a, b, temp, llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, temp=temp, v_chunks=chunks), rows)
    again = x.clone()
    _check_grad(x, t, a, b, temp, llc.llc_token_logprobs_grad(again, t, a, grad_entropy=b, temp=temp, out={"grad": again}), rows)
    s = llc.llc_token_logprobs(x, t, 0, temp=temp, want_lse=True)
    _check_grad(x, t, a, b, temp, llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, temp=temp, lse=s["lse"], entropy=s["entropy"]), rows)


# the mean's weights: few enough that one multiply-add an entry forms the gradient; with them the entropy's; weights too large for that
WEIGHTS = {"mean": (1.0, 0.0), "entropy": (1.0, 0.3), "large": (100.0, 0.0), "large, entropy": (100.0, 30.0)}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(20, 61), (20, 1030), (20, 9001), (20, 40003), (90, 70001)])
@pytest.mark.parametrize("weights", WEIGHTS)
def test_gradient_where_a_NaN_lies_among_numbers(R, V, dtype, weights):
    x = _rows(R, V, dtype, V)
    t = torch.randint(0, V, (R, 3), generator=_gen(V), device=DEV).to(torch.int32)
    for r in range(R):
        x[r, (41 * r) % V] = float("nan")
        if r % 2 == 0:
            x[r, V - 1] = float("nan")
    t[:, 0] = (torch.arange(R, device=DEV) * 41) % V  # (a token without mass)
    x[3, ::7] = float("nan")
    x[4, ::2] = -float("inf")
    x[5, 1::2] = float("inf")
    size, bonus = WEIGHTS[weights]
    a = size * torch.rand(R, 3, generator=_gen(1), device=DEV) / R
    b = torch.full((R,), bonus / R, device=DEV) if bonus else None
    _gradients(x, t, a, b, 1.0, slice(0, 20))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [61, 1030, 9001, 40003, 70001])
@pytest.mark.parametrize("weights", WEIGHTS)
def test_gradient_beside_signalling_NaNs(V, dtype, weights):
    x = _with_signalling(V, dtype)
    if V > 65536:
        x = torch.cat([x] * 5)  # (so many that a row is a workgroup's)
    R = x.shape[0]
    t = torch.randint(0, V, (R, 5), generator=_gen(V), device=DEV).to(torch.int32)
    t[:, 0] = (torch.arange(R, device=DEV) % 20 * 37) % (V - 2) + 1
    t[:, 1] = t[:, 0] - 1
    size, bonus = WEIGHTS[weights]
    a = size * torch.rand(R, 5, generator=_gen(1), device=DEV) / R
    b = torch.full((R,), bonus / R, device=DEV) if bonus else None
    _gradients(x, t, a, b, 0.8, slice(0, 20))


MASKS = [1e9, -1e9, -3e9, 1e10, -1e10, -3e10, 1e20, -1e20, 1e30, -1e30]


def _large(V, dtype, temp):
    """Rows that begin with, or are, large finite values, and rows around the size where they stop to be told by fp32 products."""
    x = _rows(3 * len(MASKS) + 8, V, dtype, V)
    noise = _rows(8, V, F32, V + 1)
    for i, mask in enumerate(MASKS):
        x[3 * i, : V - V // 3] = mask          # a block before the others
        x[3 * i + 1] = mask                    # nothing else: uniform
        x[3 * i + 2] = mask * (1.0 + 1e-3 * noise[0].abs()).to(dtype)
    edge = 2.0 ** 22 * temp / 1.4426950408889634
    steps = torch.linspace(-40, 40, V, device=DEV)
    for i, row in enumerate((edge + steps, edge - steps, -edge + steps, -edge - steps, edge / 2 + noise[1], -edge / 2 + noise[2], 4 * edge + noise[3], noise[4] * edge)):
        x[3 * len(MASKS) + i] = row.to(dtype)
    return x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [300, 9001, 70001])
@pytest.mark.parametrize("temp", [0.7, 1.0, 2.0])
def test_scores_of_large_finite_values(temp, V, dtype):
    x = _large(V, dtype, temp)
    R = x.shape[0]
    t = torch.randint(0, V, (R, 4), generator=_gen(V), device=DEV).to(torch.int32)
    t[:, 0], t[:, 1] = 0, V - 1
    for chunks in (0, 1, 5):
        ref.check_scores(llc.llc_token_logprobs(x, t, 10, temp=temp, want_lse=True, v_chunks=chunks), x, t, 10, temp)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [300, 9001, 40003, 70001])
@pytest.mark.parametrize("temp,weights", [(0.7, "mean"), (1.0, "entropy"), (1.0, "large"), (2.0, "large, entropy")])
def test_gradient_of_large_finite_values(temp, weights, V, dtype):
    x = _large(V, dtype, temp)
    rows = slice(0, x.shape[0])
    if V > 65536:
        x = torch.cat([x] * 3)
    R = x.shape[0]
    t = torch.randint(0, V, (R, 4), generator=_gen(V), device=DEV).to(torch.int32)
    t[:, 0], t[:, 1] = 0, V - 1
    size, bonus = WEIGHTS[weights]
    a = size * torch.rand(R, 4, generator=_gen(1), device=DEV) / R
    b = torch.full((R,), bonus / R, device=DEV) if bonus else None
    _gradients(x, t, a, b, temp, rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V,chunks", [(600, 128256, 0), (90, 152064, 0), (1, 1 << 20, 1), (1, 1 << 22, 1), (2, (1 << 25) + 77, 1)])
def test_sums_of_long_rows_of_equal_entries(R, V, chunks, dtype):
    # equal terms round alike in all lanes, so that what running sums lose does not average out; the value is no power of two
    x = torch.full((R, V), -1.3, device=DEV).to(dtype)
    x[:, 5] = 0.25
    t = torch.zeros(R, 2, dtype=torch.int32, device=DEV)
    t[:, 1] = 5
    out = llc.llc_token_logprobs(x, t, 0, want_lse=True, v_chunks=chunks)
    ref.check_scores({k: v[:1] for k, v in out.items()}, x[:1], t[:1], 0, 1.0)
    for v in out.values():
        assert torch.equal(v, v[:1].expand_as(v))
    if chunks == 0:  # (the gradient's pass over rows that stay on the chip)
        a = torch.full((R, 2), 0.1, device=DEV)
        out = llc.llc_token_logprobs_grad(x, t, a)
        ref.check_scores({k: out[k][:1] for k in ("logp", "entropy")}, x[:1], t[:1], 0, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_in_place_of_a_single_row_of_any_stride(dtype):
    # the stride of one row says nothing: the transpose of a column has (1, 1)
    V = 5003
    x = _rows(V, 1, dtype, 1).t()
    t, a = torch.tensor([[7, V - 1]], dtype=torch.int32, device=DEV), torch.tensor([[0.5, -0.2]], device=DEV)
    want = llc.llc_token_logprobs_grad(x.clone(), t, a)["grad"]
    for temp_x in (x.clone().t().contiguous().t(), torch.cat([x, x])[:1]):
        lse = llc.llc_token_logprobs(temp_x, t, 0, want_lse=True)["lse"]
        other = temp_x.t().clone().t()
        assert torch.equal(llc.llc_token_logprobs_grad(temp_x, t, a, out={"grad": temp_x})["grad"], want)
        assert llc.llc_token_logprobs_grad(other, t, a, lse=lse, out={"grad": other})["grad"].shape == (1, V)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [300, 9001, 40003])
@pytest.mark.parametrize("size,temp", [(1e30, 1.0), (1e33, 1.0), (1e36, 1.0), (0.1, 1e-33), (1e-3, 2.0 ** -126), (1e-32, 1.0), (1e-32, 1e-3)])
def test_gradient_with_weights_of_all_sizes(size, temp, V, dtype):
    x = _rows(6, V, dtype, V) * temp
    x[1] = 1.5                                      # uniform
    x[2, 3:] = -float("inf")
    x[3, V // 2] = 60.0 * temp                      # p of the others down to 2^-90
    x[4, V // 2] = 110.0 * temp                     # and below 2^-126
    t = torch.randint(0, V, (6, 4), generator=_gen(V), device=DEV).to(torch.int32)
    t[:, 0] = V // 2
    a = size * torch.rand(6, 4, generator=_gen(1), device=DEV)
    for b in (None, size * torch.rand(6, generator=_gen(2), device=DEV)):
        _gradients(x, t, a, b, temp, slice(0, 6))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temp", [2.0 ** -126, 1e-30, 1e-10, 3e38])
@pytest.mark.parametrize("V", [300, 40003, 70001])
def test_scores_at_extreme_temperatures(V, temp, dtype):
    x = _rows(4, V, dtype, V)
    x[1, ::2] = 7.0
    x[2] = -1.25
    x[3, 5:] = -float("inf")
    t = torch.randint(0, V, (4, 4), generator=_gen(V), device=DEV).to(torch.int32)
    t[:, 0], t[:, 1] = 0, V - 1
    for chunks in (0, 1, 5):
        ref.check_scores(llc.llc_token_logprobs(x, t, 10, temp=temp, want_lse=True, v_chunks=chunks), x, t, 10, temp)
    a = torch.full((4, 4), temp if temp < 1 else 0.1, device=DEV)
    _gradients(x, t, a, None, temp, slice(0, 4))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(86, 127999), (86, 128000), (128, 152064), (129, 152064), (86, 262143), (90, 262144), (86, 524288)])
def test_scores_and_gradient_where_rows_begin_to_be_split_in_two(R, V, dtype):
    x = _rows(R, V, dtype, R + V)
    t = torch.randint(0, V, (R, 2), generator=_gen(V), device=DEV).to(torch.int32)
    for M in (0, 40):
        out = llc.llc_token_logprobs(x, t, M, temp=0.8, want_lse=True)
        for rows in (slice(0, 4), slice(R - 4, R)):
            ref.check_scores({k: v[rows] for k, v in out.items()}, x[rows], t[rows], M, 0.8)
    a = torch.rand(R, 2, generator=_gen(1), device=DEV) / R
    _gradients(x, t, a, None, 0.8, slice(R - 4, R))
