"""The embedding's gradient for tokens of any shape (needs an MI355X)."""
import pytest
import torch

import paper_2506_05632_amd as llc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("shape", [(), (1,), (3, 1), (2, 3, 4), (2, 1, 3, 2, 2), (0,), (2, 0, 3)])
def test_gradient_of_tokens_of_any_shape(shape):
    # what the lookup takes, its gradient takes: a single token without a dimension too
    table = torch.arange(50 * 33, device=DEV, dtype=torch.float32).view(50, 33)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    t = torch.randint(-1, 51, shape, generator=g, device=DEV).to(torch.int32)
    out = llc.llc_embed(table, t)["out"]
    grad = llc.llc_embed_grad(out, t, 50)["grad"]  # (whole numbers: sums are exact)
    times = torch.bincount(t[(t >= 0) & (t < 50)].view(-1).long(), minlength=50).view(50, 1)
    assert torch.equal(grad, table * times)
    assert torch.equal(llc.llc_embed_grad(out, t, 50, out=table.clone(), add=True)["grad"], table * (times + 1))
    with pytest.raises(ValueError):
        llc.llc_embed_grad(out.unsqueeze(0), t, 50)
    with pytest.raises(ValueError):
        llc.llc_embed_grad(torch.zeros((), device=DEV), t, 50)


def test_lookup_outputs_that_cannot_be_taken():
    table = torch.arange(50 * 6, device=DEV, dtype=torch.float32).view(50, 6)
    t = torch.tensor([[1, 2, 3], [4, 50, -1]], dtype=torch.int32, device=DEV)
    for out in (torch.empty((), device=DEV), torch.empty(2, 3, 0, device=DEV), torch.empty(36, device=DEV), torch.empty(3, 2, 6, device=DEV).transpose(0, 1),
                torch.empty(2, 6, 3, device=DEV).transpose(1, 2), torch.empty(2, 4, 6, device=DEV)[:, :3]):
        with pytest.raises(ValueError):
            llc.llc_embed(table, t, out=out)
    want = llc.llc_embed(table, t)["out"]
    for out in (torch.empty(2, 3, 6, device=DEV), torch.empty(2, 3, 9, device=DEV)[:, :, :6], torch.empty(1, 3, 2, 6, device=DEV)[0].view(2, 3, 6)):
        assert torch.equal(llc.llc_embed(table, t, out=out)["out"], want)
    assert llc.llc_embed(table, t[:0], out=torch.empty(0, 3, 6, device=DEV))["out"].shape == (0, 3, 6)
    for none in (lambda: llc.llc_embed(torch.empty(50, 0, device=DEV), t), lambda: llc.llc_embed_grad(torch.empty(2, 3, 0, device=DEV), t, 50),
                 lambda: llc.llc_embed(torch.empty(0, 6, device=DEV), t)):
        with pytest.raises(llc.LlcError) as e:
            none()
        assert e.value.code == -2
