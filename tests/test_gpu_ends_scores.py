"""Scores of tokens and their gradient against 64-bit evaluations on the host (needs an MI355X)."""
import numpy as np
import pytest
import torch

import ends_util as ref
import paper_2506_05632_amd as llc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
LOWEST = {F32: torch.finfo(F32).min, BF16: torch.finfo(BF16).min}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(R, V, dtype, seed, scale=2.0, pad=0, offset=0):
    x = scale * torch.randn(R, offset + V + pad, generator=_gen(seed), device=DEV)
    return x.to(dtype)[:, offset:offset + V]


def _tokens(R, G, V, seed):
    t = torch.randint(-1, V + 1, (R, G), generator=_gen(seed + 1), device=DEV)  # (-1: empty, V: outside)
    return t.to(torch.int32)


SIZES = [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 257, 1000, 2047, 4099, 8191, 16385, 32000, 50257, 128256]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", SIZES)
def test_scores_of_every_length(V, dtype):
    R = 3
    for G, M, temp in ((1, 1, 1.0), (5, 50, 0.7), (70, 128, 1.3)):
        x, t = _rows(R, V, dtype, 10 * V + G), _tokens(R, G, V, V)
        out = llc.llc_token_logprobs(x, t, M, temp=temp, want_lse=True)
        ref.check_scores(out, x, t, M, temp)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(1, 128256), (2, 152064), (17, 32000), (130, 9000), (300, 4100), (700, 1000), (2000, 513)])
def test_scores_of_few_and_many_rows(R, V, dtype):
    x, t = _rows(R, V, dtype, R + V), _tokens(R, 2, V, R)
    ref.check_scores(llc.llc_token_logprobs(x, t, 20, want_lse=True), x, t, 20, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v_chunks", [1, 2, 3, 7, 16, 64])
def test_scores_do_not_depend_on_the_split(v_chunks, dtype):
    for R, V in ((3, 50257), (2, 1500), (2, 5)):
        x, t = _rows(R, V, dtype, V), _tokens(R, 4, V, 3)
        ref.check_scores(llc.llc_token_logprobs(x, t, 30, temp=0.9, want_lse=True, v_chunks=v_chunks), x, t, 30, 0.9)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [5, 300, 9001, 70001])
def test_masks_infinities_and_rows_without_mass(V, dtype):
    inf, nan = float("inf"), float("nan")
    x = _rows(12, V, dtype, V).clone()
    x[0] = -inf                                        # nothing at all
    x[1] = -inf; x[1, V - 1] = 0.5                     # one entry at the end
    x[2] = LOWEST[dtype]                               # masked by the lowest value throughout: uniform
    x[3] = LOWEST[dtype]; x[3, V // 2] = -3.0          # all but one
    x[4] = nan; x[4, 0] = 1.0
    x[5] = inf                                         # no mass, not all of it
    x[6, ::2] = inf; x[6, 1::4] = nan
    x[7, : V - V // 3] = -inf
    x[8] = nan
    x[9] = 7.25                                        # all equal
    x[10, : V // 2] = -0.0; x[10, V // 2:] = 0.0       # zeros of either sign are equal
    x[11, 1::2] = LOWEST[dtype]
    t = _tokens(12, 6, V, 5)
    t[:, 0] = 0
    t[:, 1] = V - 1
    for temp in (1.0, 0.01, 30.0):
        for chunks in (0, 1, 5):
            out = llc.llc_token_logprobs(x, t, 40, temp=temp, want_lse=True, v_chunks=chunks)
            ref.check_scores(out, x, t, 40, temp)
            assert not torch.isnan(out["logp"]).any() and not torch.isnan(out["top_logp"]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_values_far_from_zero(dtype):
    # the distance between entries is what counts: 2^-23 of it, not of the values
    V = 30011
    for shift, scale in ((3000.0, 1.0), (-20000.0, 3.0), (0.0, 300.0), (1e30, 1e28)):
        x = (_rows(4, V, F32, 1, scale=scale) + shift).to(dtype)
        t = _tokens(4, 3, V, 2)
        want = ref.scores(x, t, 10, 0.8)
        out = llc.llc_token_logprobs(x, t, 10, temp=0.8, want_lse=True)
        ref.close(out["logp"], want["logp"], ref.SUM, 2 * ref.STEP)
        ref.close(out["entropy"], want["entropy"], 2 * ref.SUM, 2 * ref.SUM)
        np.testing.assert_array_equal(out["top_ids"].cpu().numpy(), want["top_ids"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "two values", "last tile"])
def test_orders_that_offer_every_entry(order, dtype):
    V = 40007
    ramp = torch.linspace(-6, 6, V, device=DEV)
    x = {"ascending": ramp, "descending": ramp.flip(0), "equal": torch.ones(V, device=DEV),
         "two values": (torch.arange(V, device=DEV) % 2).float(),
         "last tile": torch.where(torch.arange(V, device=DEV) >= V - 200, 3.0, -ramp.abs())}[order]
    x = x.expand(3, V).contiguous().to(dtype)
    t = _tokens(3, 1, V, 4)
    for M in (1, 31, 128):
        for chunks in (0, 1, 4):
            ref.check_scores(llc.llc_token_logprobs(x, t, M, v_chunks=chunks), x, t, M, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_alignments(dtype):
    R, V = 9, 5003
    for offset in (0, 1, 2, 3, 5):
        x = _rows(R, V, dtype, 7, pad=11, offset=offset)
        t = _tokens(R, 8, V, 6)[:, 2:5]
        ref.check_scores(llc.llc_token_logprobs(x, t, 12), x, t, 12, 1.0)
        column = _tokens(R, 8, V, 6)[:, 3]
        out = llc.llc_token_logprobs(x, column, 0, want_entropy=False)
        assert set(out) == {"logp"} and out["logp"].shape == (R,)
        ref.check_scores(out, x, column, 0, 1.0)
    x = _rows(1, V, dtype, 8).expand(R, V)  # one row for all
    t = _tokens(R, 2, V, 9)
    ref.check_scores(llc.llc_token_logprobs(x, t, 3), x, t, 3, 1.0)


def test_offsets_beyond_32_bits():
    R, V, stride = 3, 3000, 1 << 30  # (the last row starts 2^31 elements in)
    buffer = torch.empty(2 * stride + V + 1, dtype=BF16, device=DEV)
    x = buffer.as_strided((R, V), (stride, 1), 1)
    x.copy_(_rows(R, V, BF16, 3))
    t = _tokens(R, 2, V, 3)
    ref.check_scores(llc.llc_token_logprobs(x, t, 5), x, t, 5, 1.0)
    a = torch.randn(R, 2, device=DEV)
    want, tol = ref.gradient(x, t, a, None, 1.0)
    out = llc.llc_token_logprobs_grad(x, t, a, out={"grad": x})["grad"]
    assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()


def test_log_weights_take_no_temperature():
    x, t = _rows(4, 700, F32, 1), _tokens(4, 2, 700, 1)
    ref.check_scores(llc.llc_token_logprobs(x, t, 3, kind="logw", temp=5.0), x, t, 3, 1.0)


def test_no_tokens_and_no_rows():
    x = _rows(4, 700, F32, 1)
    out = llc.llc_token_logprobs(x, None, 3)
    assert "logp" not in out
    ref.check_scores(out, x, None, 3, 1.0)
    out = llc.llc_token_logprobs(x[:0], torch.empty(0, 2, dtype=torch.int32, device=DEV), 3)
    assert out["logp"].shape == (0, 2) and out["top_ids"].shape == (0, 3)
    assert llc.llc_token_logprobs_grad(x[:0], None, None)["grad"].shape == (0, 700)
    g = llc.llc_token_logprobs_grad(x, None, None)["grad"]
    assert torch.count_nonzero(g) == 0


def test_the_lists_are_those_of_the_truncated_coupling():
    # coupling the lists gives what coupling the truncated rows gives
    R, V, M, K = 64, 9000, 50, 4
    target = _rows(R, V, F32, 1)
    draft = target + 0.5 * _rows(R, V, F32, 2)
    lists = [llc.llc_token_logprobs(x, None, M) for x in (draft, target)]
    got = llc.llc_couple_topm(lists[0]["top_ids"], lists[0]["top_logp"], lists[1]["top_ids"], lists[1]["top_logp"], K, kind="logw", seed=5)
    cut = [torch.full_like(x, -float("inf")).scatter(1, l["top_ids"].long(), l["top_logp"]) for x, l in ((draft, lists[0]), (target, lists[1]))]
    want = llc.llc_couple(cut[0], cut[1], K, kind="logw", seed=5)
    assert torch.equal(got["X"], want["X"]) and torch.equal(got["Y"], want["Y"])


def test_another_stream_and_a_graph():
    x, t = _rows(8, 20000, BF16, 1), _tokens(8, 3, 20000, 1)
    a = torch.randn(8, 3, device=DEV)
    want, want_grad = llc.llc_token_logprobs(x, t, 9), llc.llc_token_logprobs_grad(x, t, a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = llc.llc_token_logprobs(x, t, 9)
    side.synchronize()
    for name in want:
        assert torch.equal(got[name], want[name]), name
    still, still_t = x.clone(), t.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = llc.llc_token_logprobs(still, still_t, 9)
        held_grad = llc.llc_token_logprobs_grad(still, still_t, a)
    for n in range(4):
        still.copy_(x.roll(n, 0))
        still_t.copy_(t.roll(n, 0))
        graph.replay()
        torch.cuda.synchronize()
        now, now_grad = llc.llc_token_logprobs(still, still_t, 9), llc.llc_token_logprobs_grad(still, still_t, a)
        for name in now:
            assert torch.equal(held[name], now[name]), (n, name)
        assert torch.equal(held_grad["grad"], now_grad["grad"]), n


# ---- the gradient

def _check_grad(x, t, a, b, temp, out, grad):
    want, tol = ref.gradient(x, t, a, b, temp)
    far = np.abs(grad.detach().cpu().double().numpy() - want) - tol
    assert far.max() <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))
    if out is not None:
        ref.check_scores(out, x, t, 0, temp)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", SIZES)
def test_gradient_of_every_length(V, dtype):
    R = 3
    for G, temp, bonus in ((1, 1.0, False), (5, 0.7, True), (70, 1.3, True)):
        x, t = _rows(R, V, dtype, 10 * V + G), _tokens(R, G, V, V)
        a = torch.randn(R, G, generator=_gen(V), device=DEV)
        b = torch.randn(R, generator=_gen(V + 1), device=DEV) if bonus else None
        out = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, temp=temp)
        _check_grad(x, t, a, b, temp, out, out["grad"])
        # from what the forward call returned, into a wider buffer whose other columns stay
        scores = llc.llc_token_logprobs(x, t, 0, temp=temp, want_lse=True)
        wide = torch.full((R, V + 9), 77.0, dtype=dtype, device=DEV)
        llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, temp=temp, lse=scores["lse"], entropy=scores["entropy"],
                                    out={"grad": wide[:, 5:5 + V]})
        _check_grad(x, t, a, b, temp, None, wide[:, 5:5 + V])
        assert (wide[:, :5] == 77).all() and (wide[:, 5 + V:] == 77).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(1, 152064), (17, 32000), (130, 9000), (300, 70001), (700, 1000)])
def test_gradient_of_few_and_many_rows(R, V, dtype):
    x, t = _rows(R, V, dtype, R + V), _tokens(R, 2, V, R)
    a, b = torch.randn(R, 2, generator=_gen(1), device=DEV), torch.randn(R, generator=_gen(2), device=DEV)
    out = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b)
    _check_grad(x, t, a, b, 1.0, out, out["grad"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [5, 300, 9001, 70001])
def test_gradient_of_masked_rows(V, dtype):
    inf, nan = float("inf"), float("nan")
    x = _rows(10, V, dtype, V).clone()
    x[0] = -inf
    x[1] = -inf; x[1, V - 1] = 0.5
    x[2] = LOWEST[dtype]
    x[3] = LOWEST[dtype]; x[3, V // 2] = -3.0
    x[4] = nan; x[4, 0] = 1.0
    x[5] = inf
    x[6, ::2] = inf; x[6, 1::4] = nan
    x[7, : V - V // 3] = -inf
    x[8] = 7.25
    t = _tokens(10, 6, V, 5)
    t[:, 0] = 0
    t[:, 1] = V - 1
    t[:, 2] = V - 1  # (the same token twice)
    a, b = torch.randn(10, 6, generator=_gen(1), device=DEV), torch.randn(10, generator=_gen(2), device=DEV)
    a[t < 0] = nan   # (not looked at)
    a[t >= V] = inf
    for temp in (1.0, 0.05):
        for chunks in (0, 1, 3):
            out = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, temp=temp, v_chunks=chunks)
            assert not torch.isnan(out["grad"]).any()
            _check_grad(x, t, a, b, temp, out, out["grad"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(4, 3001), (3, 128256), (300, 5000)])
def test_gradient_in_place(R, V, dtype):
    x, t = _rows(R, V, dtype, 3, pad=3), _tokens(R, 4, V, 3)
    a = torch.randn(R, 4, generator=_gen(4), device=DEV)
    want = llc.llc_token_logprobs_grad(x, t, a)["grad"]
    scores = llc.llc_token_logprobs(x, t, 0, want_lse=True)
    again = x.clone()
    got = llc.llc_token_logprobs_grad(again, t, a, out={"grad": again})["grad"]
    assert got.data_ptr() == again.data_ptr() and torch.equal(got, want)
    again = x.clone()
    got = llc.llc_token_logprobs_grad(again, t, a, lse=scores["lse"], out={"grad": again})["grad"]
    _check_grad(x, t, a, None, 1.0, None, got)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [4, 6, 1023, 1024, 1025, 1031, 4096, 4097, 8192, 8195, 16384, 16391, 32768, 32775, 40003, 65536, 65543])
def test_gradient_where_a_row_takes_one_more_tile(V, dtype):
    R = 3
    for G, pad in ((2, 0), (300, 3), (1100, 5)):  # (more tokens than a wavefront, and than a workgroup)
        x, t = _rows(R, V, dtype, V + G, pad=pad, offset=pad // 2), _tokens(R, G, V, V)
        t[:, -1] = V - 1
        a, b = torch.randn(R, G, generator=_gen(V), device=DEV), torch.randn(R, generator=_gen(V + 1), device=DEV)
        wide = torch.full((R, V + 2 * pad), 77.0, dtype=dtype, device=DEV)
        out = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b)
        _check_grad(x, t, a, b, 1.0, out, out["grad"])
        llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, out={"grad": wide[:, pad:pad + V]})
        assert torch.equal(wide[:, pad:pad + V], out["grad"])
        assert (wide[:, :pad] == 77).all() and (wide[:, pad + V:] == 77).all()
        again = x.clone()
        assert torch.equal(llc.llc_token_logprobs_grad(again, t, a, grad_entropy=b, out={"grad": again})["grad"], out["grad"])


@pytest.mark.parametrize("R,V,dtype", [(90, 66001, F32), (90, 100003, F32), (87, 131072, BF16), (90, 140001, BF16), (86, 200003, BF16), (86, 49153, F32)])
def test_gradient_of_many_long_rows(R, V, dtype):
    inf = float("inf")
    x, t = _rows(R, V, dtype, V).clone(), _tokens(R, 3, V, V)
    x[1] = -inf
    x[2] = LOWEST[dtype]
    x[3] = -inf; x[3, V - 1] = 1.0
    x[4, : V - 700] = -inf
    x[5, ::3] = inf; x[5, 1::3] = float("nan")
    x[6, 500:] = LOWEST[dtype]
    t[:, 0] = V - 1
    a, b = torch.randn(R, 3, generator=_gen(1), device=DEV), torch.randn(R, generator=_gen(2), device=DEV)
    out = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b)
    _check_grad(x[:12], t[:12], a[:12], b[:12], 1.0, {k: v[:12] for k, v in out.items()}, out["grad"][:12])
    _check_grad(x[-2:], t[-2:], a[-2:], b[-2:], 1.0, {k: v[-2:] for k, v in out.items()}, out["grad"][-2:])
    few = llc.llc_token_logprobs_grad(x[:4], t[:4], a[:4], grad_entropy=b[:4])  # (split over more workgroups)
    _check_grad(x[:4], t[:4], a[:4], b[:4], 1.0, few, few["grad"])
    again = x.clone()
    assert torch.equal(llc.llc_token_logprobs_grad(again, t, a, grad_entropy=b, out={"grad": again})["grad"], out["grad"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,V", [(1, 47999), (1, 48000), (5, 63999), (5, 64000), (85, 50001), (86, 50001), (85, 64001), (86, 64001), (4, 300007)])
def test_scores_where_rows_begin_to_be_split(R, V, dtype):
    x, t = _rows(R, V, dtype, R + V), _tokens(R, 300 if R < 6 else 2, V, R)
    ref.check_scores(llc.llc_token_logprobs(x, t, 40, temp=0.8, want_lse=True), x, t, 40, 0.8)


def test_the_longest_row():
    V = 2 ** 31 - 5
    x = torch.full((1, V), -float("inf"), dtype=BF16, device=DEV)
    places = [0, 5, V // 2, V - 1030, V - 1025, V - 9, V - 2, V - 1]
    values = torch.tensor([0.5, -1.0, 2.0, 1.0, 0.25, -2.0, 3.0, 1.5], dtype=BF16)
    x[0, places] = values.to(DEV)
    small = values.float().view(1, -1)  # (the same row without what has no mass)
    t = torch.tensor([[V - 1, 0, -1, V - 1030]], dtype=torch.int32, device=DEV)
    a, b = torch.tensor([[0.5, -1.0, 2.0, 0.25]], device=DEV), torch.tensor([0.7], device=DEV)
    for chunks in (0, 1):
        out = llc.llc_token_logprobs(x, t, 10, want_lse=True, v_chunks=chunks)
        ref.check_scores({k: out[k] for k in ("entropy", "lse")}, small, None, 0, 1.0)
        order = torch.argsort(values.float(), descending=True)
        assert out["top_ids"][0].tolist() == [places[i] for i in order] + [-1, -1]
        lp = torch.log_softmax(values.double(), 0)
        assert (out["logp"][0].cpu().double() - torch.stack([lp[7], lp[0], lp.new_zeros(()), lp[3]])).abs().max() < 1e-5
    want, tol = ref.gradient(small, torch.tensor([[7, 0, -1, 3]]), a.cpu(), b.cpu(), 1.0)
    got = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, out={"grad": x})["grad"]
    assert torch.count_nonzero(got) == 8
    assert (np.abs(got[0, places].cpu().double().numpy() - want[0]) <= tol[0] + ref.OUT[BF16] * np.abs(want[0])).all()


def test_gradient_against_differences():
    # f(x + h v) - f(x - h v) over 2 h for directions v of length one: the third derivative of these sums is below
    # 2 (|a| + |b| (1 + ln V)) / T^3, and f is known to 2e-6 of its weights, so h = 2^-5 leaves 3e-4 of them
    R, V, G, T, h = 5, 900, 3, 0.9, 2.0 ** -5
    x, t = _rows(R, V, F32, 1), torch.randint(0, V, (R, G), generator=_gen(2), device=DEV, dtype=torch.int32)
    a, b = torch.randn(R, G, generator=_gen(3), device=DEV), torch.randn(R, generator=_gen(4), device=DEV)
    grad = llc.llc_token_logprobs_grad(x, t, a, grad_entropy=b, temp=T)["grad"].double()

    def f(x):
        s = llc.llc_token_logprobs(x, t, 0, temp=T)
        return (s["logp"].double() * a).sum(1) + s["entropy"].double() * b

    size = a.double().abs().sum(1) + b.double().abs() * (1 + np.log(V))
    top = x.argmax(dim=1)
    for n in range(12):
        v = torch.randn(R, V, generator=_gen(10 + n), device=DEV)
        if n >= 8:  # along the entries that matter
            v = torch.zeros_like(v)
            v[torch.arange(R), t[:, n % G].long() if n % 2 else top] = 1.0
        v = v / v.norm(dim=1, keepdim=True)
        got = (f(x + h * v) - f(x - h * v)) / (2 * h)
        bound = size * (2 * h * h / 6 / T ** 3 + 2 * 4e-6 / (2 * h)) + 1e-5
        assert ((got - (grad * v).sum(1)).abs() <= bound).all(), n


def test_refusals():
    x, t = _rows(4, 100, F32, 1), _tokens(4, 2, 100, 1)
    a = torch.zeros(4, 2, device=DEV)
    for bad in (lambda: llc.llc_token_logprobs(x.cpu(), t), lambda: llc.llc_token_logprobs(x, t.long()), lambda: llc.llc_token_logprobs(x.half(), t),
                lambda: llc.llc_token_logprobs(x, t[:3]), lambda: llc.llc_token_logprobs(x.t(), t), lambda: llc.llc_token_logprobs(x, t, kind="probs"),
                lambda: llc.llc_token_logprobs(x, t.cpu()), lambda: llc.llc_token_logprobs(x[0], t), lambda: llc.llc_token_logprobs_grad(x, t, None),
                lambda: llc.llc_token_logprobs_grad(x, t, a.double()), lambda: llc.llc_token_logprobs_grad(x, t, a[:, :1]),
                lambda: llc.llc_token_logprobs_grad(x, t, a, grad_entropy=a), lambda: llc.llc_token_logprobs_grad(x, t, a, lse=a[:, 0]),
                lambda: llc.llc_token_logprobs_grad(x, t, a, out={"grad": x.bfloat16()})):
        with pytest.raises(ValueError):
            bad()
    for code, bad in ((-2, lambda: llc.llc_token_logprobs(x, t, 129)), (-3, lambda: llc.llc_token_logprobs(x, t, temp=0.0)),
                      (-6, lambda: llc.llc_token_logprobs(x, t, 3, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))),
                      (-8, lambda: llc.llc_token_logprobs(x, t, v_chunks=65)),
                      (-1, lambda: llc.llc_token_logprobs_grad(x, t, a, grad_entropy=a[:, 0].contiguous(), lse=torch.zeros(4, 2, dtype=torch.float64, device=DEV))),
                      (-2, lambda: llc.llc_token_logprobs_grad(x, t, a, out={"grad": torch.zeros(100, device=DEV).expand(4, 100)}))):
        with pytest.raises(llc.LlcError) as e:
            bad()
        assert e.value.code == code


def test_refusals_of_outputs_and_workspaces():
    x, t = _rows(4, 100, F32, 1), _tokens(4, 2, 100, 1)
    a = torch.zeros(4, 2, device=DEV)
    f32 = lambda *shape: torch.zeros(shape, device=DEV)  # noqa: E731
    for out in ({"logp": f32(4)}, {"logp": f32(2, 4).t()}, {"logp": f32(4, 2).double()}, {"logp": torch.zeros(4, 2)},
                {"logp": f32(4, 2), "entropy": f32(3)}, {"logp": f32(4, 2), "lse": f32(4, 2)}, {"logp": f32(4, 2), "top_ids": f32(4, 3), "top_logp": f32(4, 3)}):
        with pytest.raises(ValueError):
            llc.llc_token_logprobs(x, t, 3, out=out)
    for out in ({"grad": f32(4, 100), "logp": f32(4)}, {"grad": f32(4, 100), "entropy": f32(4, 1)}, {"grad": f32(4, 99)}, {"grad": torch.zeros(4, 100)}):
        with pytest.raises(ValueError):
            llc.llc_token_logprobs_grad(x, t, a, out=out)
    for workspace in (torch.zeros(1 << 16, dtype=torch.uint8), f32(1 << 14), torch.zeros(1 << 17, dtype=torch.uint8, device=DEV)[::2]):
        for bad in (lambda: llc.llc_token_logprobs(x, t, workspace=workspace), lambda: llc.llc_token_logprobs_grad(x, t, a, workspace=workspace),
                    lambda: llc.llc_embed_grad(x, t[:, 0], 9, workspace=workspace), lambda: llc.llc_clip_grad_norm([x], 1.0, workspace=workspace)):
            with pytest.raises(ValueError):
                bad()
    with pytest.raises(llc.LlcError) as e:
        llc.llc_token_logprobs(x, t, 3, out={"entropy": f32(4)})
    assert e.value.code == -1


def test_a_dry_run_writes_nothing():
    x, t = _rows(4, 100, F32, 1), _tokens(4, 2, 100, 1)
    grad = torch.full((4, 100), 5.0, device=DEV)
    llc.llc_token_logprobs_grad(x, t, torch.ones(4, 2, device=DEV), out={"grad": grad}, flags=llc.FLAG_DRY_RUN)
    out = llc.llc_token_logprobs(x, t, 2, out={"logp": torch.full((4, 2), 5.0, device=DEV), "top_ids": torch.full((4, 2), 5, dtype=torch.int32, device=DEV),
                                               "top_logp": torch.full((4, 2), 5.0, device=DEV)}, flags=llc.FLAG_DRY_RUN)
    torch.cuda.synchronize()
    assert (grad == 5).all() and all((v == 5).all() for v in out.values())
