"""Host-side checks of the calls at the vocabulary's two ends: struct layout and argument errors (no GPU)."""
import ctypes
import os
import subprocess

import pytest

import paper_2506_05632_amd as llc
from paper_2506_05632_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"llc_token_logprobs_args": binding.TokenLogprobsArgs, "llc_token_logprobs_grad_args": binding.TokenLogprobsGradArgs,
           "llc_embed_args": binding.EmbedArgs, "llc_embed_grad_args": binding.EmbedGradArgs,
           "llc_clip_grad_norm_args": binding.ClipGradNormArgs}


def test_every_field_lies_where_the_binding_has_it(tmp_path):
    lines = []
    for name, struct in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {field}));' for field, _ in struct._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "llc.h"\nint main(void){\n' + "\n".join(lines)
                   + "\nreturn LLC_TOP_MAX == %d ? 0 : 1;}\n" % binding.TOP_MAX)
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for struct in STRUCTS.values():
        want += [ctypes.sizeof(struct)] + [getattr(struct, field).offset for field, _ in struct._fields_]
    assert got == want


def _filled(struct, base, kw):
    a = struct()
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


SCORES = dict(R=4, V=64, G=2, M=3, dtype=0, kind=0, x=0x1000, stride_r=64, temp=1.0, tokens=0x2000, tok_stride_r=2, logp=0x3000, entropy=0x3000,
              top_ids=0x3000, top_logp=0x3000, workspace=0x4000, workspace_bytes=1 << 20)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(tokens=None), -1), (dict(logp=None), -1), (dict(top_ids=None), -1), (dict(top_logp=None), -1),
    (dict(R=-1), -2), (dict(R=1 << 24), -2), (dict(V=0), -2), (dict(V=(1 << 31) - 4), -2), (dict(G=-1), -2), (dict(G=65536), -2),
    (dict(M=-1), -2), (dict(M=129), -2), (dict(stride_r=-1), -2), (dict(tok_stride_r=-1), -2),
    (dict(temp=0.0), -3), (dict(temp=float("nan")), -3), (dict(temp=float("inf")), -3),
    (dict(dtype=2), -4), (dict(kind=1), -4), (dict(kind=7), -4),
    (dict(x=0x1002), -5), (dict(tokens=0x2002), -5),
    (dict(workspace=None), -6), (dict(workspace=0x4010), -6), (dict(workspace_bytes=300), -6),
    (dict(flags=1), -8), (dict(v_chunks=65), -8), (dict(v_chunks=-1), -8),
    (dict(flags=4), 0), (dict(flags=4, G=0, tokens=None, logp=None), 0), (dict(flags=4, M=0, top_ids=None, top_logp=None), 0),
    (dict(flags=4, kind=2, temp=0.0), 0), (dict(R=0, x=None), 0),
])
def test_scores_arguments(kw, code):
    lib = llc.load()
    assert lib.llc_token_logprobs(ctypes.byref(_filled(binding.TokenLogprobsArgs, SCORES, kw))) == code
    assert lib.llc_token_logprobs(None) == -1


GRAD = dict(R=4, V=64, G=2, dtype=0, kind=0, x=0x1000, stride_r=64, temp=1.0, tokens=0x2000, tok_stride_r=2, grad_logp=0x2000, grad_logp_stride_r=2,
            grad=0x8000, grad_stride_r=64, workspace=0x4000, workspace_bytes=1 << 20)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(grad=None), -1), (dict(tokens=None), -1), (dict(grad_logp=None), -1), (dict(lse_in=0x6000, grad_entropy=0x6000), -1),
    (dict(V=0), -2), (dict(R=-1), -2), (dict(grad_stride_r=63), -2), (dict(grad_logp_stride_r=-1), -2), (dict(stride_r=-1), -2),
    (dict(grad=0x1000, grad_stride_r=65), -2),
    (dict(temp=-1.0), -3), (dict(dtype=3), -4), (dict(kind=1), -4),
    (dict(grad=0x8001), -5), (dict(grad_logp=0x2001), -5),
    (dict(workspace=None), -6), (dict(workspace_bytes=100), -6),
    (dict(flags=2), -8), (dict(v_chunks=65), -8), (dict(lse_in=0x6000, logp=0x7000), -8), (dict(lse_in=0x6000, lse=0x7000), -8),
    (dict(lse_in=0x6000, entropy=0x7000), -8),
    (dict(flags=4), 0), (dict(flags=4, lse_in=0x6000, workspace=None), 0), (dict(flags=4, grad=0x1000), 0), (dict(R=0, x=None, grad=None), 0),
])
def test_gradient_of_scores_arguments(kw, code):
    lib = llc.load()
    assert lib.llc_token_logprobs_grad(ctypes.byref(_filled(binding.TokenLogprobsGradArgs, GRAD, kw))) == code
    assert lib.llc_token_logprobs_grad(None) == -1


EMBED = dict(T=4, N=10, D=8, dtype=0, out_dtype=1, table=0x1000, table_stride_n=8, tokens=0x2000, tok_stride=1, scale=1.0, out=0x3000, out_stride_t=8)


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), -1), (dict(tokens=None), -1), (dict(out=None), -1),
    (dict(T=-1), -2), (dict(N=0), -2), (dict(D=0), -2), (dict(D=1 << 31), -2), (dict(table_stride_n=-1), -2), (dict(out_stride_t=7), -2),
    (dict(tok_stride=-1), -2), (dict(dtype=2), -4), (dict(out_dtype=-1), -4), (dict(table=0x1002), -5), (dict(out=0x3001), -5), (dict(tokens=0x2001), -5),
    (dict(scale=float("nan")), -8), (dict(flags=16), -8), (dict(flags=4), 0), (dict(T=0, table=None), 0),
])
def test_lookup_arguments(kw, code):
    lib = llc.load()
    assert lib.llc_embed(ctypes.byref(_filled(binding.EmbedArgs, EMBED, kw))) == code
    assert lib.llc_embed(None) == -1


EMBED_GRAD = dict(T=4, N=10, D=8, dtype=0, grad_dtype=1, g=0x1000, g_stride_t=8, tokens=0x2000, tok_stride=1, scale=1.0, grad=0x3000, grad_stride_n=8,
                  workspace=0x4000, workspace_bytes=1 << 24)


@pytest.mark.parametrize("kw,code", [
    (dict(g=None), -1), (dict(tokens=None), -1), (dict(grad=None), -1),
    (dict(T=-1), -2), (dict(N=0), -2), (dict(N=(1 << 27) + 1), -2), (dict(D=0), -2), (dict(g_stride_t=-1), -2), (dict(grad_stride_n=7), -2),
    (dict(tok_stride=-1), -2), (dict(dtype=2), -4), (dict(grad_dtype=5), -4), (dict(g=0x1001), -5), (dict(grad=0x3001), -5),
    (dict(workspace=None), -6), (dict(workspace=0x4008), -6), (dict(workspace_bytes=8), -6),
    (dict(scale=float("inf")), -8), (dict(flags=32), -8), (dict(flags=4), 0), (dict(flags=4, add=1), 0), (dict(T=0, add=1, grad=None), 0),
])
def test_gradient_of_lookup_arguments(kw, code):
    lib = llc.load()
    assert lib.llc_embed_grad(ctypes.byref(_filled(binding.EmbedGradArgs, EMBED_GRAD, kw))) == code
    assert lib.llc_embed_grad(None) == -1


def _clip(grads=(0x1000, 0x2000), numel=(8, 9), dtype=(0, 1), out=None, **kw):
    n = len(grads)
    arrays = [(ctypes.c_void_p * n)(*grads), (ctypes.c_int64 * n)(*numel), (ctypes.c_int32 * n)(*dtype)]
    a = binding.ClipGradNormArgs()
    a.n = n
    a.grads, a.numel, a.dtype = (ctypes.cast(v, ctypes.c_void_p) for v in arrays)
    if out is not None:
        arrays.append((ctypes.c_void_p * n)(*out))
        a.out = ctypes.cast(arrays[-1], ctypes.c_void_p)
    a.max_norm, a.norm, a.workspace, a.workspace_bytes = 1.0, 0x3000, 0x4000, 1 << 20
    for k, v in kw.items():
        setattr(a, k, v)
    return llc.load().llc_clip_grad_norm(ctypes.byref(a))


@pytest.mark.parametrize("kw,code", [
    (dict(norm=None), -1), (dict(grads=(0x1000, None)), -1), (dict(out=(None, 0x2000)), -1),
    (dict(n=-1), -2), (dict(n=(1 << 20) + 1), -2), (dict(numel=(-1, 3)), -2), (dict(numel=(1 << 40, 1)), -2),
    (dict(dtype=(0, 2)), -4), (dict(grads=(0x1002, 0x2000)), -5), (dict(out=(0x1000, 0x2001)), -5), (dict(norm=0x3001), -5),
    (dict(workspace=None), -6), (dict(workspace_bytes=8), -6), (dict(max_norm=0.0), -8), (dict(max_norm=float("nan")), -8), (dict(flags=1), -8),
    (dict(flags=4), 0), (dict(flags=4, max_norm=float("inf")), 0), (dict(flags=4, grads=(0x1000, None), numel=(8, 0)), 0),
])
def test_clipping_arguments(kw, code):
    assert _clip(**kw) == code
    assert llc.load().llc_clip_grad_norm(None) == -1


def test_workspace_sizes():
    assert llc.llc_token_logprobs_workspace_size(4, 64, 3) >= 4 * (32 + 24)
    assert llc.llc_token_logprobs_workspace_size(4, 0, 3) == 0 and llc.llc_token_logprobs_workspace_size(4, 64, 129) == 0
    assert llc.llc_embed_grad_workspace_size(4, 10, 8) > 0 and llc.llc_embed_grad_workspace_size(4, 0, 8) == 0
    assert llc.llc_clip_grad_norm_workspace_size(0) > 0 and llc.llc_clip_grad_norm_workspace_size(-1) == 0
    # what a call asks for is what it takes
    lib = llc.load()
    for R, V, M in ((1, 128256, 50), (300, 50257, 128), (1 << 20, 1000, 0)):
        n = llc.llc_token_logprobs_workspace_size(R, V, M)
        a = _filled(binding.TokenLogprobsArgs, SCORES, dict(R=R, V=V, M=M, flags=4, workspace_bytes=n))
        assert lib.llc_token_logprobs(ctypes.byref(a)) == 0
        a.v_chunks, a.workspace_bytes = 7, 7 * R * (32 + 8 * M) + 32 * R + 512
        assert lib.llc_token_logprobs(ctypes.byref(a)) == 0
    for T, N, D in ((1, 1, 1), (70000, 128256, 4096), (5, 1 << 27, 3)):
        a = _filled(binding.EmbedGradArgs, EMBED_GRAD, dict(T=T, N=N, D=D, flags=4, g_stride_t=D, grad_stride_n=D,
                                                            workspace_bytes=llc.llc_embed_grad_workspace_size(T, N, D)))
        assert lib.llc_embed_grad(ctypes.byref(a)) == 0
