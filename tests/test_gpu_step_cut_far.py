"""Cut rows whose largest entry is far over what a row's first entries show, masked rows, and the ends of what settings and numbers may be,
against 64-bit evaluations of the definition (needs an MI355X)."""
import math

import pytest
import torch

import paper_2506_05632_amd as llc
import step_util

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _spiked(V, over, apart, dtype, g):
    """Normal rows with a group of entries `over` the others' largest and `apart` from each other, at an index that no part of a row begins with."""
    x = torch.randn(3, V, generator=g, device=DEV)
    at = 70000 if V > 70000 else V - 3000
    x[:, at] = x.amax(dim=1) + over
    for i in range(1, 5):
        x[1, at + 97 * i] = x[1, at] - i * apart
    x[2, at - 1:at + 40] = x[2, at]
    return x.to(TYPES[dtype])


FAR = [(0.02, 15.0), (0.01, 8.0), (0.01, 6.0), (1e-3, 0.9), (1e-30, 1.0), (1.0, 800.0), (1.0, 730.0), (1.0, 650.0), (0.7, 3e4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp,over", FAR)
@pytest.mark.parametrize("V", [20011, 128256])
def test_uncut_rows_with_an_entry_far_over_the_others(V, temp, over, dtype):
    g = _gen(V)
    x = _spiked(V, over, 0.9 * temp, dtype, g)
    u = torch.cat([torch.tensor([0.0, 0.3, 1.0 - 2.0 ** -24], device=DEV).expand(3, 3), torch.rand(3, 5, generator=g, device=DEV)], 1)
    step_util.check_sample(llc.llc_sample(x, u, temp=temp, want_kept=True), x, u, temp=temp)
    # the same through a row's own settings, which may be none
    own = dict(temp=torch.full((3,), temp, device=DEV), top_p=torch.ones(3, device=DEV))
    step_util.check_sample(llc.llc_sample(x, u, want_kept=True, **own), x, u, **own)


def test_uncut_rows_of_log_weights_far_apart():
    x = _spiked(30011, 900.0, 0.9, "f32", _gen(1))
    u = torch.rand(3, 4, generator=_gen(2), device=DEV)
    step_util.check_sample(llc.llc_sample(x, u, kind="logw", want_kept=True), x, u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_several_pieces_a_tile(dtype):
    # over 2^20 entries; the settings take the list, the range, what is narrowed down, and the tiles
    g = _gen(51)
    V = (1 << 20) + (1 << 17) + 77
    x = torch.randn(2, V, generator=g, device=DEV)
    x[0, V - 5] = 9.0
    x[1, 1 << 20:] = -math.inf
    x = x.to(TYPES[dtype])
    u = torch.rand(2, 3, generator=g, device=DEV)
    for settings in (dict(), dict(temp=1e-3), dict(top_k=40), dict(top_k=5000), dict(top_p=0.4)):
        step_util.check_sample(llc.llc_sample(x, u, want_kept=True, **settings), x, u, **settings)
    for settings in (dict(top_k=5000), dict(min_p=0.2)):
        step_util.check_truncate(llc.llc_truncate(x, **settings), x, **settings)


SHARES = [dict(top_p=0.9), dict(top_p=0.3), dict(top_p=0.9, min_p=0.01), dict(top_p=0.5, min_p=1e-4)]


def _both(x, u, **settings):
    step_util.check_sample(llc.llc_sample(x, u, want_kept=True, **settings), x, u, **settings)
    step_util.check_truncate(llc.llc_truncate(x, **settings), x, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp,over", FAR)
@pytest.mark.parametrize("V", [20011, 128256])
def test_shares_of_rows_with_an_entry_far_over_the_others(V, temp, over, dtype):
    g = _gen(V + 1)
    x = _spiked(V, over, 0.9 * temp, dtype, g)
    u = torch.rand(3, 5, generator=g, device=DEV)
    for settings in SHARES + [dict(top_p=0.9, top_k=V), dict(top_p=0.9, top_k=3)]:
        _both(x, u, temp=temp, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temp", [1.0, 0.01, 1e-3])
@pytest.mark.parametrize("allowed", [3, 100, 1000])
def test_shares_of_rows_that_allow_a_few_entries(allowed, temp, dtype):
    # -inf but for some, as where what may follow is given: fewer than a list of a share is made for, in the sample and in all
    g = _gen(allowed)
    V = 128256
    x = torch.full((4, V), -math.inf, device=DEV)
    for r in range(4):
        at = torch.randperm(V, generator=g, device=DEV)[:allowed]
        x[r, at] = torch.randn(allowed, generator=g, device=DEV)
        x[r, at[0]] = x[r].max() + 3.0 * r
    x[3, 12345:12350] = x[3].max() - 0.4 * temp
    x = x.to(TYPES[dtype])
    u = torch.rand(4, 5, generator=g, device=DEV)
    for settings in [dict()] + SHARES:
        _both(x, u, temp=temp, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shares_of_rows_masked_by_the_least_number(dtype):
    # the same with the type's lowest value in the masked places, which has mass where nothing is over it
    g = _gen(61)
    V = 50021
    low = torch.finfo(TYPES[dtype]).min
    x = torch.full((4, V), low, device=DEV)
    x[0, 30001:30011] = torch.randn(10, generator=g, device=DEV)
    x[1, V - 1] = 1.0
    x[2, 45000::7] = 0.5 * torch.randn(x[2, 45000::7].shape, generator=g, device=DEV)
    x = x.to(TYPES[dtype])
    u = torch.rand(4, 5, generator=g, device=DEV)
    for settings in [dict(), dict(top_k=7)] + SHARES:
        _both(x, u, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [600, 5000, 128256])
def test_no_share_at_all_leaves_the_first_entry(V, dtype):
    # a row's own top_p of 0 or less, where a list would hold the row's entries and where it would not
    g = _gen(71)
    x = torch.zeros(5, V, device=DEV)
    x[1] = torch.linspace(-3.0, 3.0, V, device=DEV)
    x[2] = torch.randint(0, 3, (V,), generator=g, device=DEV).float()
    x[3] = torch.randn(V, generator=g, device=DEV)
    x[4, ::2] = -math.inf
    x = x.to(TYPES[dtype])
    u = torch.tensor([[0.0, 0.5, 1.0 - 2.0 ** -24, 1.0]], device=DEV).repeat(5, 1)
    for p in (0.0, -1.0, -math.inf):
        top_p = torch.full((5,), p, device=DEV)
        top_p[3] = 0.5
        for settings in (dict(), dict(top_k=900), dict(min_p=0.2), dict(top_k=torch.tensor([0, 0, 7, 0, 3000], dtype=torch.int32, device=DEV))):
            _both(x, u, top_p=top_p, **settings)
    first = x.float().argmax(dim=1)
    out = llc.llc_sample(x, u, top_p=torch.zeros(5, device=DEV), want_kept=True)
    assert out["kept"].tolist() == [1] * 5 and torch.equal(out["tokens"].long(), first[:, None].expand(5, 4))
    # the least positive share, as a number
    _both(x, u, top_p=1e-45)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=5000), dict(top_k=20000, min_p=1e-4), dict(top_p=0.97, temp=1.5), dict(top_k=60), dict(top_k=100000, top_p=0.999999)])
def test_one_and_more_take_the_last_kept_entry(settings, dtype):
    # rows whose ends are masked or have next to no mass: sums along them differ by roundings alone
    g = _gen(81)
    R, V = 20, 128256
    x = 1.5 * torch.randn(R, V, generator=g, device=DEV)
    for r in range(R):
        x[r, V - 700 * r - 300:] = -math.inf if r % 2 else -45.0
        x[r, 40000 + 900 * r:52000 + 800 * r] = -math.inf
    x = x.to(TYPES[dtype])
    inf = math.inf
    u = torch.tensor([[1.0, 1.0 + 2.0 ** -23, 2.0, inf, 1.0 - 2.0 ** -24, 0.0, -0.0, -1.0, -inf, math.nan]], device=DEV).repeat(R, 1)
    out = llc.llc_sample(x, u, want_kept=True, **settings)
    step_util.check_sample(out, x, u, **settings)
    cut = llc.llc_truncate(x, **settings)["logits"]
    kept = torch.isfinite(cut)
    index = torch.arange(V, device=DEV)
    last, first = torch.where(kept, index, -1).amax(dim=1), torch.where(kept, index, V).amin(dim=1)
    tokens = out["tokens"].long()
    for s in range(4):
        assert torch.equal(tokens[:, s], last), s
    assert kept.gather(1, tokens[:, :9]).all()
    assert all(torch.equal(tokens[:, s], first) for s in (5, 6, 7, 8))


def test_the_longest_row():
    # V = 2^31 - 5: places of all kinds at their widest.  Numbers in 16 bits, so that thousands of equals lie about the cut
    V = (1 << 31) - 5
    x = torch.empty(1, V, dtype=torch.bfloat16, device=DEV).normal_(generator=_gen(91))
    x[0, V - 1] = x[0, 1 << 30] = 9.0
    u = torch.tensor([[0.0, 0.3, 0.7, 1.0 - 2.0 ** -24, 1.0]], device=DEV)
    for k in (3, 5000):
        cut = llc.llc_truncate(x, top_k=k)
        kept = torch.isfinite(cut["logits"][0])
        assert cut["kept"].item() == k == int(kept.sum())
        at = kept.nonzero().view(-1)
        last = x[0, at].min()
        more = x[0] > last
        assert bool(kept[more].all()) and bool((x[0, at] >= last).all())
        n = k - int(more.sum())
        equal = (x[0] == last).nonzero().view(-1)
        assert len(equal) >= n > 0 and bool(kept[equal[:n]].all()) and not bool(kept[equal[n:]].any())
        out = llc.llc_sample(x, u, top_k=k, want_kept=True)
        upto = (x[0, at].double() - 9.0).exp().cumsum(0)
        want = at[torch.searchsorted(upto, u[0].double() * upto[-1], right=True).clamp(max=k - 1)]
        assert torch.equal(out["tokens"][0].long(), want) and out["kept"].item() == k
        logp = x[0, want].double() - 9.0 - upto[-1].log()
        assert bool(((out["logp"][0].double() - logp).abs() <= 1.01 * 2.0 ** -24 * logp.abs() + 1e-12).all())
        del cut, kept, more, equal
    # equal masses: every sum is a whole number
    x.zero_()
    out = llc.llc_sample(x, u[:, [0, 3, 4]], want_kept=True)
    assert out["tokens"][0].tolist() == [0, V - 128, V - 1] and out["kept"].item() == V
    assert bool((out["logp"].double() + math.log(V)).abs().max() <= 1.01 * 2.0 ** -24 * math.log(V) + 1e-12)
    half = torch.full((1,), 0.5, device=DEV)
    assert llc.llc_sample(x, half)["tokens"].item() == V // 2
