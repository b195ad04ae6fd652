"""Fits a small drafter to a target model, then lets it draft: the operators at the vocabulary's two ends beside the coupling.

A training step looks the contexts' tokens up (llc_embed), draws what the target says next (llc_couple, draft side alone),
takes loss and gradient of the drafter's logits in one call, in place (llc_token_logprobs_grad), adds the rows' gradients up
(llc_embed_grad) and bounds the step (llc_clip_grad_norm).  A serving step takes the likeliest tokens of both models
(llc_token_logprobs) and couples the lists (llc_couple_topm).  The drafter is then held in 4 bits (llc_quantize): it looks tokens up
(llc_embed_quantized), multiplies (llc_matvec_quantized) and goes on from what it draws of its cut rows (llc_sample), and the cut
rows of both models are coupled (llc_truncate, llc_couple).  Data are synthetic: the target is a random bigram model.

    python examples/fit_drafter.py [--steps 300]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_05632_amd as llc  # noqa: E402


class Target:
    """Next-token logits of a random model that looks at the last token alone."""

    def __init__(self, V, rank, gen, device):
        self.left = torch.randn(V, rank, generator=gen, device=device)
        self.right = 2.5 * torch.randn(rank, V, generator=gen, device=device) / rank ** 0.5

    def logits(self, context):
        return llc.llc_embed(self.left, context)["out"] @ self.right


class Drafter:
    """Embedding, one hidden layer, output layer; gradients are written into the parameters' .grad."""

    def __init__(self, V, D, gen, device):
        self.scale = D ** 0.5
        self.table = torch.randn(V, D, generator=gen, device=device) * 0.1 / self.scale
        self.hidden = torch.randn(D, D, generator=gen, device=device) / D ** 0.5
        self.head = torch.randn(D, V, generator=gen, device=device) / D ** 0.5
        self.params = [self.table, self.hidden, self.head]

    def logits(self, context):
        h = llc.llc_embed(self.table, context, scale=self.scale)["out"]
        z = torch.relu(h @ self.hidden)
        return h, z, z @ self.head

    def step(self, context, following, optimizer, most):
        """One step on the mean of -ln p(following | context); that mean, and the gradient's norm."""
        h, z, logits = self.logits(context)
        weight = torch.full(following.shape, -1.0 / following.numel(), device=logits.device)
        logp = torch.empty(following.shape, device=logits.device)
        g = llc.llc_token_logprobs_grad(logits, following, weight, out={"grad": logits, "logp": logp})["grad"]  # (of the loss)
        gz = (g @ self.head.t()) * (z > 0)
        self.head.grad = z.t() @ g
        self.hidden.grad = h.t() @ gz
        self.table.grad = llc.llc_embed_grad(gz @ self.hidden.t(), context, self.table.shape[0], scale=self.scale)["grad"]
        norm = llc.llc_clip_grad_norm([p.grad for p in self.params], most)["norm"]
        optimizer.step()
        return -logp.mean(), norm


class Served:
    """A drafter with its three layers in 4 bits, `group` entries of a row to a scale."""

    def __init__(self, drafter, group=32):
        self.scale, self.group = drafter.scale, group
        self.D = drafter.table.shape[1]
        # rows of tokens as they are looked up; of the others' a row for each of the outputs
        self.table, self.hidden, self.head = (llc.llc_quantize(w, group=group, zeros=True, scales_dtype=torch.float32)
                                              for w in (drafter.table, drafter.hidden.t().contiguous(), drafter.head.t().contiguous()))

    def product(self, x, layer):
        return llc.llc_matvec_quantized(x, layer["codes"], layer["scales"], zeros=layer["zeros"], group=self.group)["out"]

    def logits(self, context):
        h = llc.llc_embed_quantized(self.table["codes"], self.table["scales"], context, self.D, zeros=self.table["zeros"], group=self.group, scale=self.scale,
                                    out_dtype=torch.float32)["out"]
        z = torch.relu(self.product(h, self.hidden))
        return h, z, self.product(z, self.head)

    def text(self, context, u, **cuts):
        """Tokens [R,L] that follow the contexts' [R], each drawn with its own of u [R,L] and looked up for the next."""
        tokens = []
        for n in range(u.shape[1]):
            context = llc.llc_sample(self.logits(context)[2], u[:, n:n + 1], want_logp=False, **cuts)["tokens"].view(-1)
            tokens.append(context)
        return torch.stack(tokens, 1)


def accepted_cut(target, drafter, context, K, seed, **cuts):
    """The same share by whole rows, both sides cut."""
    rows = [llc.llc_truncate(x, want_kept=False, **cuts)["logits"] for x in (drafter.logits(context)[2], target.logits(context))]
    return llc.llc_couple(rows[0], rows[1], K, seed=seed)["accept"].float().mean()


def accepted(target, drafter, context, M, K, seed):
    """Share of the contexts whose next token is among the K drafts, both sides cut to their M likeliest."""
    lists = [llc.llc_token_logprobs(x, None, M, want_entropy=False) for x in (drafter.logits(context)[2], target.logits(context))]
    out = llc.llc_couple_topm(lists[0]["top_ids"], lists[0]["top_logp"], lists[1]["top_ids"], lists[1]["top_logp"], K, kind="logw", seed=seed)
    return out["accept"].float().mean()


def run(steps=300, V=2000, D=64, rank=16, batch=1024, M=50, K=4, seed=0, device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    target, drafter = Target(V, rank, gen, device), Drafter(V, D, gen, device)
    optimizer = torch.optim.Adam(drafter.params, lr=1e-2)
    probe = torch.randint(0, V, (batch,), generator=gen, device=device, dtype=torch.int32)
    floor = llc.llc_token_logprobs(target.logits(probe), None)["entropy"].mean().item()  # no drafter's loss is below it
    before = accepted(target, drafter, probe, M, K, seed).item()
    losses = []
    for n in range(steps):
        context = torch.randint(0, V, (batch,), generator=gen, device=device, dtype=torch.int32)
        following = llc.llc_couple(target.logits(context), None, 1, seed=seed + 1 + n, flags=llc.FLAG_DRAFT_ONLY)["X"].view(-1)
        losses.append(drafter.step(context, following, optimizer, 1.0))
    after = accepted(target, drafter, probe, M, K, seed).item()
    served = Served(drafter)
    text = served.text(probe[:4], torch.rand(4, 16, generator=gen, device=device), top_k=M, top_p=0.95)
    in_4_bits = accepted(target, served, probe, M, K, seed).item(), accepted_cut(target, served, probe, K, seed, top_k=M).item()
    return {"loss": [float(loss) for loss, _ in losses], "norm": [float(norm) for _, norm in losses], "entropy": floor,
            "accepted": (before, after), "accepted_in_4_bits": in_4_bits, "text": text}


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=300)
    found = run(parser.parse_args().steps)
    print("loss %.3f -> %.3f (the target's entropy: %.3f)" % (found["loss"][0], found["loss"][-1], found["entropy"]))
    print("accepted with 4 drafts: %.3f -> %.3f" % found["accepted"])
    print("the same with layers in 4 bits: %.3f of lists, %.3f of cut rows" % found["accepted_in_4_bits"])
