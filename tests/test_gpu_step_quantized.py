"""Layers in 4 bits against 64-bit evaluations of their definitions (needs an MI355X)."""
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


def _layer(N, D, group, scales, zeros, g, pad=0):
    """Random codes and scales of a layer, in buffers with `pad` more columns."""
    groups = -(-D // group)
    codes = torch.randint(0, 256, (N, (D + 1) // 2 + pad), generator=g, device=DEV, dtype=torch.uint8)[:, :(D + 1) // 2]
    s = (0.01 + 0.02 * torch.rand(N, groups + pad, generator=g, device=DEV)).to(TYPES[scales])[:, :groups]
    z = torch.randint(0, 16, (N, groups + pad), generator=g, device=DEV, dtype=torch.uint8)[:, :groups] if zeros else None
    return codes, s, z


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scales", ["f32", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize(group, zeros, scales, dtype):
    for N, D in ((1, 1), (3, 7), (5, 31), (2, 128), (17, 129), (4, 512), (9, 1537), (3, 2048), (2, 5001)):
        w = (torch.randn(N, D, generator=_gen(D), device=DEV) * 0.02).to(TYPES[dtype])
        out = llc.llc_quantize(w, group=group, zeros=zeros, scales_dtype=TYPES[scales])
        step_util.check_quantize(out, w, group, zeros, TYPES[scales])


@pytest.mark.parametrize("scales", ["f32", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_borders(zeros, scales):
    # ties (halves of the largest entry), one sign only, nothing at all, the smallest and largest numbers, what is not finite
    inf, nan = math.inf, math.nan
    base = torch.tensor([1.0, 0.5, -0.5, 0.25, 7.0, 3.5, -3.5, 1.5], device=DEV)
    rows = [base.repeat(8), base.abs().repeat(8) + 2.0, -base.abs().repeat(8) - 1.0, torch.zeros(64, device=DEV), base.repeat(8) * 2.0 ** -149,
            base.repeat(8) * 2.0 ** -130, base.repeat(8) * 2.0 ** 125, torch.full((64,), nan, device=DEV), torch.full((64,), inf, device=DEV)]
    mixed = base.repeat(8).clone()
    mixed[3], mixed[10], mixed[40] = nan, inf, -inf
    extreme = torch.full((64,), 3.4e38, device=DEV)
    extreme[1::2] = -3.4e38
    w = torch.stack(rows + [mixed, extreme, torch.arange(64, device=DEV) * 1.0, torch.full((64,), -0.0, device=DEV)])
    for group in (32, 64):
        out = llc.llc_quantize(w, group=group, zeros=zeros, scales_dtype=TYPES[scales])
        step_util.check_quantize(out, w, group, zeros, TYPES[scales])


def test_quantize_into_given_rows():
    N, D = 6, 200
    w = torch.randn(N, D + 9, generator=_gen(1), device=DEV)[:, 4:4 + D]
    codes = torch.full((N, 111), 0xEE, dtype=torch.uint8, device=DEV)
    scales = torch.full((N, 6), -1.0, device=DEV)
    zeros = torch.full((N, 5), 99, dtype=torch.uint8, device=DEV)
    out = llc.llc_quantize(w, group=64, zeros=True, scales_dtype=torch.float32, out={"codes": codes[:, 3:103], "scales": scales[:, 1:5], "zeros": zeros[:, 1:]})
    step_util.check_quantize(out, w, 64, True, torch.float32)
    assert (codes[:, :3] == 0xEE).all() and (codes[:, 103:] == 0xEE).all() and (scales[:, 0] == -1).all() and (scales[:, 5] == -1).all() and (zeros[:, 0] == 99).all()
    step_util.check_quantize(llc.llc_quantize(w[0:1].expand(4, D)), w[0:1].expand(4, D), 128, False, torch.bfloat16)
    assert llc.llc_quantize(w[:0])["codes"].shape == (0, 100)


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scales", ["f32", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_embed(group, zeros, scales, out_dtype):
    for N, D in ((1, 1), (50, 7), (300, 64), (33, 129), (20, 1537), (7, 4096)):
        g = _gen(D)
        codes, s, z = _layer(N, D, group, scales, zeros, g, pad=3)
        tokens = torch.randint(-2, N + 2, (3, 11), generator=g, device=DEV, dtype=torch.int32)
        out = llc.llc_embed_quantized(codes, s, tokens, D, zeros=z, group=group, scale=3.0, out_dtype=TYPES[out_dtype])["out"]
        t = tokens.cpu().numpy()
        w = step_util.values(codes, s, z, D, group)
        want = np.where(((t >= 0) & (t < N))[..., None], 3.0 * w[np.clip(t, 0, N - 1)], 0.0)
        # two products in fp32 and the output's rounding
        tol = np.abs(want) * (2 * 2.0 ** -24 + 1.01 * step_util.STEP[TYPES[out_dtype]])
        assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()


def test_embed_outputs_and_tokens():
    N, D = 40, 100
    codes, s, z = _layer(N, D, 32, "f32", True, _gen(2))
    tokens = torch.randint(0, N, (12, 5), generator=_gen(3), device=DEV, dtype=torch.int32)
    want = llc.llc_embed_quantized(codes, s, tokens, D, zeros=z, group=32)["out"]
    assert want.shape == (12, 5, D) and want.dtype == torch.float32
    turned = llc.llc_embed_quantized(codes, s, tokens.t(), D, zeros=z, group=32)["out"]
    assert torch.equal(turned, want.transpose(0, 1))
    buffer = torch.full((12, D + 7), 5.0, device=DEV)
    llc.llc_embed_quantized(codes, s, tokens[:, 2], D, zeros=z, group=32, out=buffer[:, 3:3 + D])
    assert torch.equal(buffer[:, 3:3 + D], want[:, 2]) and (buffer[:, :3] == 5).all() and (buffer[:, 3 + D:] == 5).all()
    assert llc.llc_embed_quantized(codes, s, tokens[:0], D, zeros=z, group=32)["out"].shape == (0, 5, D)
    one = llc.llc_embed_quantized(codes, s, torch.tensor(7, dtype=torch.int32, device=DEV), D, zeros=z, group=32)["out"]
    assert one.shape == (D,)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scales", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_matvec(group, scales, dtype):
    for R, N, D in ((1, 1, 1), (1, 16, 128), (2, 17, 31), (3, 33, 130), (1, 100, 2048), (5, 50, 1537), (16, 64, 256), (17, 48, 300), (33, 40, 512), (48, 129, 96),
                    (64, 20, 1000), (65, 35, 260), (130, 18, 640)):
        g = _gen(R * 1000 + D)
        codes, s, z = _layer(N, D, group, scales, (R + N) % 2 == 1, g)
        x = torch.randn(R, D, generator=g, device=DEV).to(TYPES[dtype])
        for out_dtype in TYPES.values():
            out = llc.llc_matvec_quantized(x, codes, s, zeros=z, group=group, out_dtype=out_dtype)["out"]
            step_util.check_matvec(out, x, codes, s, z, group)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,N,D", [(1, 2000, 9000), (1, 40, 40000), (9, 5000, 4096), (64, 700, 8192), (40, 33000, 200), (61, 3000, 2050), (2, 70000, 64)])
def test_matvec_of_every_plan(R, N, D, dtype):
    # one wavefront a tile, several; x in LDS at once, in parts; several tiles a workgroup
    g = _gen(N)
    codes, s, z = _layer(N, D, 64, "bf16", True, g)
    x = torch.randn(R, D, generator=g, device=DEV).to(TYPES[dtype])
    step_util.check_matvec(llc.llc_matvec_quantized(x, codes, s, zeros=z, group=64, out_dtype=torch.float32)["out"], x, codes, s, z, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_matvec_of_unlike_inputs(dtype):
    # far from the mean, channels that outweigh the others, tiny and large numbers, zeros
    g = _gen(21)
    R, N, D = 6, 70, 700
    codes, s, z = _layer(N, D, 128, "f32", False, g)
    x = torch.randn(R, D, generator=g, device=DEV)
    x[0] += 30.0
    x[1, ::97] *= 1e4
    x[2] *= 1e-30
    x[3] *= 1e30
    x[4] = 0.0
    x[5] = 1.0
    x = x.to(TYPES[dtype])
    step_util.check_matvec(llc.llc_matvec_quantized(x, codes, s, out_dtype=torch.float32)["out"], x, codes, s, None, 128)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_matvec_strides_and_rows_that_are_not_finite(dtype):
    g = _gen(22)
    R, N, D = 9, 45, 333
    codes, s, z = _layer(N, D, 32, "bf16", True, g, pad=5)
    wide = torch.randn(R, D + 11, generator=g, device=DEV).to(TYPES[dtype])
    x = wide[:, 5:5 + D]
    want = llc.llc_matvec_quantized(x.contiguous(), codes.contiguous(), s.contiguous(), zeros=z.contiguous(), group=32, out_dtype=torch.float32)["out"]
    step_util.check_matvec(want, x, codes, s, z, 32)
    buffer = torch.full((R, N + 6), 5.0, device=DEV)
    llc.llc_matvec_quantized(x, codes, s, zeros=z, group=32, out=buffer[:, 1:1 + N])
    assert torch.equal(buffer[:, 1:1 + N], want) and (buffer[:, 0] == 5).all() and (buffer[:, 1 + N:] == 5).all()
    same = llc.llc_matvec_quantized(x[3:4].expand(4, D), codes, s, zeros=z, group=32, out_dtype=torch.float32)["out"]
    assert torch.equal(same, want[3:4].expand(4, N))
    x[2, 7], x[5, 100] = math.inf, math.nan
    got = llc.llc_matvec_quantized(x, codes, s, zeros=z, group=32, out_dtype=torch.float32)["out"]
    others = [r for r in range(R) if r not in (2, 5)]
    assert torch.equal(got[others], want[others]) and not torch.isfinite(got[[2, 5]]).any()
    assert llc.llc_matvec_quantized(x[:0], codes, s, zeros=z, group=32)["out"].shape == (0, N)


def test_the_same_bits_again_on_a_stream_and_from_a_graph():
    g = _gen(23)
    w = torch.randn(3000, 1024, generator=g, device=DEV) * 0.02
    x = torch.randn(20, 1024, generator=g, device=DEV)
    tokens = torch.randint(0, 3000, (64,), generator=g, device=DEV, dtype=torch.int32)

    def all_of_them():
        q = llc.llc_quantize(w, group=64, zeros=True)
        return [*q.values(), llc.llc_embed_quantized(q["codes"], q["scales"], tokens, 1024, zeros=q["zeros"], group=64)["out"],
                llc.llc_matvec_quantized(x, q["codes"], q["scales"], zeros=q["zeros"], group=64)["out"]]

    want = all_of_them()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        again = all_of_them()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = all_of_them()
    first = w.clone()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(caught, want))
        w.mul_(-0.7)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(caught, all_of_them()))
        w.copy_(first)


def test_the_longest_rows():
    # 33 rows of 2^27 in 32 bits: x as it is laid out has more than 2^31 pieces of 16 bytes.  Ones in few places, scales powers of two: every sum is exact
    R, N, D, G = 33, 5, 1 << 27, 128
    g = torch.Generator(device=DEV).manual_seed(2)
    codes = torch.randint(0, 256, (N, D // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.full((N, D // G), 0.25, device=DEV)
    scales[:, ::3] = 2.0
    x = torch.zeros(R, D, device=DEV)
    at = torch.cat([torch.tensor([0, 1, D // 2 + 5, D - 128, D - 1]), torch.randint(0, D, (60,), generator=torch.Generator().manual_seed(3))]).unique().to(DEV)
    x[:, at] = torch.randint(-2, 3, (R, len(at)), generator=g, device=DEV).float()
    out = llc.llc_matvec_quantized(x, codes, scales, group=G)["out"]
    byte = codes[:, at // 2].long()
    q = torch.where(at % 2 == 0, byte & 15, byte >> 4).double() - 8.0
    want = x[:, at].double() @ (q * scales[:, at // G].double()).t()
    assert torch.equal(out.double(), want)
