"""A drafting step from end to end: lookup and products in 4 bits, cut rows, sampling, coupling (needs an MI355X)."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2506_05632_amd as llc
import step_util

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fit_drafter.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("fit_drafter", EXAMPLE)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _served(example, V, D, group, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return example.Served(example.Drafter(V, D, gen, DEV), group)


@pytest.mark.parametrize("V,D,group,R", [(2000, 64, 32, 5), (1537, 130, 64, 33), (4099, 256, 128, 1)])
def test_every_part_of_a_step(example, V, D, group, R):
    served = _served(example, V, D, group)
    context = torch.randint(0, V, (R,), device=DEV, dtype=torch.int32)
    h, z, logits = served.logits(context)
    table = step_util.values(served.table["codes"], served.table["scales"], served.table["zeros"], D, group)
    want = torch.from_numpy(table)[context.long().cpu()] * served.scale
    # a product of a scale and a whole number, and one with the table's scale: a rounding each, and that of the scale's own to 32 bits
    assert ((h.cpu().double() - want).abs() <= 3.1 * 2.0 ** -24 * want.abs()).all()
    for x, layer, out in ((h, served.hidden, served.product(h, served.hidden)), (z, served.head, logits)):
        step_util.check_matvec(out, x, layer["codes"], layer["scales"], layer["zeros"], group)
    u = torch.rand(R, 3, device=DEV)
    for cuts in (dict(top_k=50, top_p=0.95), dict(top_p=0.8), dict(min_p=0.3)):
        step_util.check_sample(llc.llc_sample(logits, u, want_kept=True, **cuts), logits, u, **cuts)
        step_util.check_truncate(llc.llc_truncate(logits, **cuts), logits, **cuts)


def test_what_is_coupled_is_among_the_kept(example):
    served = _served(example, 2000, 64, 32)
    context = torch.randint(0, 2000, (64,), device=DEV, dtype=torch.int32)
    logits = served.logits(context)[2]
    target = logits + 0.5 * torch.randn(logits.shape, device=DEV)
    draft, cut = llc.llc_truncate(logits, top_k=20)["logits"], llc.llc_truncate(target, top_p=0.3)["logits"]
    out = llc.llc_couple(draft, cut, 4, seed=3)
    assert torch.isfinite(draft.gather(1, out["X"].long())).all() and torch.isfinite(cut.gather(1, out["Y"].long().view(-1, 1))).all()
    # Algorithm 2 over the same cut rows, the drafts of a step as its tokens
    S, L, K, V = 8, 1, 4, 2000
    rows = cut.view(S, 8, V)[:, :2].unsqueeze(2).expand(S, L + 1, K, V).contiguous()
    tokens = llc.llc_couple(draft.view(S, 8, V)[:, 0].contiguous(), None, K, seed=5, flags=llc.FLAG_DRAFT_ONLY)["X"].view(S, L, K)
    found = llc.llc_verify(rows, tokens, seed=5)
    first = found["Y"][:, 0].long()
    assert torch.isfinite(rows[:, 0, 0].gather(1, first.view(-1, 1))).all()


@pytest.mark.parametrize("R", [2, 20])
def test_a_step_captured_twice_and_replayed(example, R):
    # two graphs of the same step, each with workspaces of its own, replayed in turn with eager steps between
    served = _served(example, 1500, 128, 64, seed=1)
    side = torch.cuda.Stream()
    contexts = [torch.randint(0, 1500, (R,), device=DEV, dtype=torch.int32) for _ in range(2)]
    us = [torch.rand(R, 4, device=DEV) for _ in range(2)]
    cuts = dict(top_k=30, top_p=0.9)
    served.text(contexts[0], us[0], **cuts)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for context, u in zip(contexts, us):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(served.text(context, u, **cuts))
        graphs.append(graph)
    for turn in range(3):
        for context, u in zip(contexts, us):
            context.copy_(torch.randint(0, 1500, (R,), device=DEV, dtype=torch.int32))
            u.uniform_()
        for graph in graphs:
            graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = [served.text(context, u, **cuts) for context, u in zip(contexts, us)]
        torch.cuda.current_stream().wait_stream(side)
        for out, want in zip(outs, again):
            assert torch.equal(out, want) and (out >= 0).all()


def test_the_example_serves_in_4_bits(example):
    found = example.run(steps=3)
    assert all(0.0 <= share <= 1.0 for share in found["accepted_in_4_bits"])
    assert found["text"].shape == (4, 16) and int(found["text"].min()) >= 0 and int(found["text"].max()) < 2000
    assert all(math.isfinite(loss) for loss in found["loss"])
