"""Sampling and cut rows against 64-bit evaluations of their definition (needs an MI355X)."""
import math

import numpy as np
import pytest
import torch

import paper_2506_05632_amd as llc
import step_util

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _zipf(R, V, steep, dtype, g):
    """Rows whose masses fall as a power of the rank, in random order, with noise."""
    x = -steep * torch.log1p(torch.rand(R, V, generator=g, device=DEV).mul(V).floor())
    return (x + 0.5 * torch.randn(R, V, generator=g, device=DEV)).to(dtype)


def _both(x, u, **settings):
    step_util.check_sample(llc.llc_sample(x, u, want_kept=True, **settings), x, u, **settings)
    step_util.check_truncate(llc.llc_truncate(x, **settings), x, **settings)


CUTS = [dict(), dict(top_k=1), dict(top_k=5), dict(top_k=40, top_p=0.9), dict(top_p=0.9), dict(top_p=0.5), dict(min_p=0.05), dict(min_p=1.0),
        dict(top_k=300, min_p=0.01), dict(top_k=20, top_p=0.8, min_p=0.1), dict(top_p=0.95, min_p=0.2), dict(top_k=700), dict(top_k=900, top_p=0.99),
        dict(top_k=1000, min_p=1e-4), dict(top_k=800, top_p=0.9, min_p=1e-3), dict(top_p=0.999)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 511, 513, 1000, 4097, 32000])
def test_every_cut(V, dtype):
    g = _gen(V)
    x = _zipf(6, V, 1.3, TYPES[dtype], g)
    u = torch.rand(6, 3, generator=g, device=DEV)
    for settings in CUTS:
        _both(x, u, temp=0.8, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steep", [0.3, 1.05, 2.5])
def test_large_vocabulary(steep, dtype):
    g = _gen(11)
    x = _zipf(5, 128256, steep, TYPES[dtype], g)
    u = torch.rand(5, 4, generator=g, device=DEV)
    for settings in (dict(), dict(top_p=0.9), dict(top_p=0.9, temp=0.7), dict(top_k=50), dict(top_k=5000, top_p=0.95), dict(min_p=0.05), dict(top_k=512, top_p=0.9)):
        _both(x, u, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_with_settings_of_their_own(dtype):
    g = _gen(3)
    R, V = 64, 5000
    x = _zipf(R, V, 1.2, TYPES[dtype], g)
    u = torch.rand(R, generator=g, device=DEV)
    settings = dict(temp=0.3 + torch.rand(R, generator=g, device=DEV), top_k=torch.randint(-1, 900, (R,), generator=g, device=DEV, dtype=torch.int32),
                    top_p=0.5 + 0.7 * torch.rand(R, generator=g, device=DEV), min_p=0.3 * torch.rand(R, generator=g, device=DEV) - 0.1)
    nan = float("nan")
    settings["temp"][:6] = torch.tensor([0.0, -1.0, nan, math.inf, 1e-38, 1e30], device=DEV)
    settings["top_p"][6:10] = torch.tensor([nan, 0.0, -3.0, math.inf], device=DEV)
    settings["min_p"][10:13] = torch.tensor([nan, 7.0, math.inf], device=DEV)
    _both(x, u, **settings)
    for name in settings:  # one of them for every row, the others numbers
        _both(x, u, **{name: settings[name]})


def test_entries_without_mass():
    inf, nan = math.inf, math.nan
    rows = [[nan, inf, -inf, nan, inf], [nan, 1.0, inf, 1.0, -inf], [-inf, -inf, -inf, -inf, 3.0], [0.0, -0.0, 0.0, -0.0, nan],
            [3.4e38, -3.4e38, 0.0, 3.4e38, nan], [1e-45, -1e-45, 0.0, inf, 0.0]]
    for dtype in TYPES.values():
        x = torch.tensor(rows, device=DEV).to(dtype)
        if dtype == torch.bfloat16:
            x[4] = torch.tensor([3.3e38, -3.3e38, 0.0, 3.3e38, nan])
        u = torch.tensor([[0.0, 0.3, 0.5, 0.74, 0.999]], device=DEV).repeat(len(rows), 1)
        for settings in (dict(), dict(top_k=1), dict(top_k=3), dict(top_p=0.5), dict(min_p=0.5), dict(top_k=2, top_p=0.6, min_p=0.1), dict(temp=1e-30), dict(temp=1e30, top_p=0.7)):
            _both(x, u, **settings)


@pytest.mark.parametrize("V", [4096, 5003, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_entries_go_by_index(V, dtype):
    # all equal; two values; few values: cuts fall among equals
    g = _gen(V + 1)
    x = torch.zeros(4, V, device=DEV)
    x[1, ::2] = -1.0
    x[2] = torch.randint(0, 8, (V,), generator=g, device=DEV).float() * -0.5
    x[3, V // 2:] = 2.0
    x = x.to(TYPES[dtype])
    u = torch.tensor([[0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24]], device=DEV).repeat(4, 1)
    for settings in (dict(), dict(top_p=0.5), dict(top_p=0.75), dict(top_k=10), dict(top_k=3000), dict(top_k=V - 1), dict(top_k=3000, top_p=0.5), dict(min_p=0.9), dict(min_p=0.9, top_p=0.3)):
        _both(x, u, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orders_that_crowd_the_kept_entries(dtype):
    # sorted vocabularies put all that is likely into the first wavefront's entries, a stride into one thread's
    V = 16384
    down = (-1.2 * torch.log1p(torch.arange(V, device=DEV).float())).to(TYPES[dtype])
    stride = torch.full((V,), -9.0, device=DEV)
    stride[5::512] = torch.linspace(0, -2, V // 512, device=DEV)
    spike = torch.full((V,), -30.0, device=DEV)
    spike[V - 1] = 4.0
    x = torch.stack([down, down.flip(0), stride.to(TYPES[dtype]), spike.to(TYPES[dtype])])
    u = torch.rand(4, 9, generator=_gen(0), device=DEV)
    for settings in CUTS:
        _both(x, u, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("grid", [0.0, 0.25, 2.0])
def test_cuts_deep_in_a_row(grid, dtype):
    # thousands of entries kept, with thousands of equals about the cut, in rows whose first entries are like the others or not
    g = _gen(31)
    V = 60001
    x = 2.0 * torch.randn(5, V, generator=g, device=DEV) - 9.0
    if grid > 0:
        x = (x / grid).round() * grid
    x[1, ::3] = -math.inf
    x[2] = x[2].sort(descending=True).values
    x[3] = x[3].sort().values
    x[4, V - 1] = 9.0
    x = x.to(TYPES[dtype])
    u = torch.rand(5, 7, generator=g, device=DEV)
    for settings in (dict(top_p=0.8), dict(top_p=0.97, temp=2.5), dict(top_p=0.99, min_p=0.02), dict(top_p=0.999, temp=0.5), dict(top_k=2500), dict(top_k=30000, temp=1.3), dict(top_k=50000, min_p=1e-5)):
        _both(x, u, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("over", [3.0, 9.0, 14.0, 40.0])
def test_a_few_entries_far_over_the_others(over, dtype):
    # the first entries of each part show nothing of them, and the row looks flat
    g = _gen(41)
    V = 70003
    x = 1.5 * torch.randn(4, V, generator=g, device=DEV)
    x[:, 60001] = x.amax(dim=1) + over
    x[1, 60002] = x[1, 60001]
    x[2, 33333] = x[2, 60001] - 0.7
    x[3, 33333] = x[3, 60001] - 7.0
    x = x.to(TYPES[dtype])
    u = torch.rand(4, 5, generator=g, device=DEV)
    for settings in (dict(top_p=0.3), dict(top_p=0.9), dict(top_p=0.9, temp=0.4), dict(top_p=0.9, temp=3.0), dict(top_p=0.9999), dict(top_k=4000), dict(top_p=0.9, min_p=0.01)):
        _both(x, u, **settings)


def test_log_weights_take_no_temperature():
    x = _zipf(4, 3001, 1.5, torch.float32, _gen(5))
    u = torch.rand(4, 2, generator=_gen(6), device=DEV)
    a = llc.llc_sample(x, u, kind="logw", temp=0.0, top_p=0.9, want_kept=True)
    b = llc.llc_sample(x, u, top_p=0.9, want_kept=True)
    assert all(torch.equal(a[n], b[n]) for n in ("tokens", "logp", "kept"))
    assert torch.equal(llc.llc_truncate(x, kind="logw", temp=-3.0, top_k=4)["logits"], llc.llc_truncate(x, top_k=4)["logits"])


def test_numbers_outside_the_unit_interval():
    x = _zipf(1, 1000, 1.1, torch.float32, _gen(7)).expand(1, 1000)
    u = torch.tensor([[-1.0, 0.0, -0.0, 1.0, 2.0, math.inf, -math.inf, math.nan]], device=DEV)
    for settings in (dict(), dict(top_k=30), dict(top_p=0.99)):
        out = llc.llc_sample(x, u, want_kept=True, **settings)
        step_util.check_sample(out, x, u, **settings)
        t = out["tokens"][0].tolist()
        assert t[0] == t[1] == t[2] == t[6] and t[3] == t[4] == t[5] and t[7] == -1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_outputs(dtype):
    g = _gen(8)
    R, V = 7, 2049
    wide = _zipf(R, V + 13, 1.4, TYPES[dtype], g)
    x = wide[:, 3:3 + V]
    u = torch.rand(R, 8, generator=g, device=DEV)[:, 1:4]
    _both(x, u, top_p=0.9)
    _both(x[0:1].expand(R, V), u, top_k=9)             # one row for all
    _both(x[2:3], u[2:3], top_k=600, top_p=0.95)       # a single row
    buffer = torch.full((R, V + 5), 7.0, device=DEV, dtype=TYPES[dtype])
    out = llc.llc_truncate(x, top_p=0.8, out={"logits": buffer[:, 2:2 + V]})
    assert "kept" not in out and (buffer[:, :2] == 7).all() and (buffer[:, 2 + V:] == 7).all()
    want = llc.llc_truncate(x, top_p=0.8)["logits"]
    assert torch.equal(buffer[:, 2:2 + V], want)
    # in place, in a wider buffer
    for settings in (dict(top_p=0.8), dict(top_k=700), dict(top_k=4)):
        copy = wide.clone()
        want = llc.llc_truncate(x, **settings)["logits"]
        llc.llc_truncate(copy[:, 3:3 + V], out={"logits": copy[:, 3:3 + V]}, **settings)
        assert torch.equal(copy[:, 3:3 + V], want)
        assert torch.equal(copy[:, :3], wide[:, :3]) and torch.equal(copy[:, 3 + V:], wide[:, 3 + V:])
    given = {"tokens": torch.full((R,), -7, dtype=torch.int32, device=DEV)}
    llc.llc_sample(x, u[:, 0], out=given)
    assert torch.equal(given["tokens"], llc.llc_sample(x, u[:, 0])["tokens"])
    none = llc.llc_sample(x[:0], u[:0], want_kept=True)
    assert none["tokens"].shape == (0, 3) and llc.llc_truncate(x[:0])["logits"].shape == (0, V)
    assert llc.llc_sample(x, u[:, :0], want_kept=True, top_k=3)["kept"].tolist() == [3] * R


def test_the_same_bits_again_on_a_stream_and_from_a_graph():
    g = _gen(9)
    x = _zipf(300, 20011, 1.1, torch.float32, g)
    u = torch.rand(300, 2, generator=g, device=DEV)
    settings = [dict(top_p=0.9), dict(top_k=40), dict(top_k=3000, top_p=0.9), dict()]
    want = [(llc.llc_sample(x, u, want_kept=True, **s), llc.llc_truncate(x, **s)) for s in settings]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        again = [(llc.llc_sample(x, u, want_kept=True, **s), llc.llc_truncate(x, **s)) for s in settings]
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = [(llc.llc_sample(x, u, want_kept=True, **s), llc.llc_truncate(x, **s)) for s in settings]
    keep = x.clone(), u.clone()
    for turn in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for got in (again, caught) if turn == 0 else (caught,):
            for a, b in zip(got, want):
                for one, other in zip(a, b):
                    assert all(torch.equal(one[n], other[n]) for n in other)
        # other inputs in the graph's buffers, then the first again
        x.copy_(_zipf(300, 20011, 1.7, torch.float32, g))
        graph.replay()
        fresh = llc.llc_sample(x, u, top_k=40)
        assert torch.equal(caught[1][0]["tokens"], fresh["tokens"])
        x.copy_(keep[0])


def test_what_is_drawn_follows_the_cut_distribution():
    # the share of each token over evenly spread numbers is its mass, to within one number
    x = _zipf(1, 500, 1.0, torch.float32, _gen(13))
    S = 60000
    u = ((torch.arange(S, device=DEV) + 0.5) / S).float()[None]
    for settings in (dict(top_k=60), dict(top_p=0.8), dict(min_p=0.02), dict()):
        tokens = llc.llc_sample(x, u, **settings)["tokens"]
        kept, mass, _ = step_util.cut(x, **settings)
        share = np.where(kept, mass, 0.0)[0]
        share /= share.sum()
        count = torch.bincount(tokens[0].long(), minlength=500).cpu().numpy() / S
        # (a number in 32 bits is within 2^-25 of its place)
        assert np.abs(count - share).max() <= 1.0 / S + 2.0 ** -23
