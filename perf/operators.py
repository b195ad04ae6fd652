"""What is measured of the operators at the vocabulary's two ends: their cases, inputs, plain forms and definitions.

A serving program scores the tokens that were drawn (their log probabilities, the rows' entropy and the top
alternatives, which are also the candidate lists of the truncated coupling) and looks the tokens up in the embedding
table for the next step.  A program that fits a drafter to a target takes the scores with their gradient, sums the embedding's gradient
by token and clips all gradients by their global norm.

`run` computes an operator in its plain form, elementary torch operations in 32 bits, or, where `own` is true, by the
library's call.  `exact` evaluates its definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
MOST_ENTRIES = 1024 * 128256   # logits of the largest listed call
MOST_TABLE = 128256 * 4096     # entries of the largest listed embedding's gradient
MOST_TOKENS = 16384
MOST_GRADIENTS = 5.4e8         # entries of the largest listed set of gradients
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # scores of one serving step of a lightly loaded server: four requests, their four drafts' tokens and the target's
        dict(name="scores_step", op="scores", R=4, V=32000, G=5, M=5, dtype="bf16", temp=1.0, masked=0.0, pad=0),
        # an ordinary batch, one token a row and twenty alternatives
        dict(name="scores_batch", op="scores", R=256, V=32000, G=1, M=20, dtype="bf16", temp=1.0, masked=0.0, pad=0),
        # an odd vocabulary under a grammar that leaves a tenth of it, rows of a wider buffer
        dict(name="scores_masked", op="scores", R=300, V=50257, G=1, M=8, dtype="f32", temp=0.8, masked=0.9, pad=31),
        # the full batch on a large vocabulary: eight drafts' tokens, the target's, and the lists of fifty for the truncated coupling
        dict(name="scores_lists", op="scores", R=1024, V=128256, G=9, M=50, dtype="f32", temp=0.7, masked=0.0, pad=0),
        # a training step of a small drafter: the negative log likelihood's gradient
        dict(name="scores_grad_nll", op="scores_grad", R=2048, V=32000, G=1, dtype="bf16", temp=1.0, entropy=False, pad=0),
        # reinforcement of the drafts' tokens by their acceptance, with an entropy bonus, on a large vocabulary
        dict(name="scores_grad_policy", op="scores_grad", R=768, V=128256, G=8, dtype="f32", temp=0.7, entropy=True, pad=0),
        # the lookup of one drafting step: eight requests with four drafts each
        dict(name="embed_step", op="embed", T=32, N=32000, D=2048, dtype="bf16", out="bf16", scale=1.0),
        # the lookup of a training batch, scaled by the root of the width, master weights in 32 bits
        dict(name="embed_train", op="embed", T=16384, N=128256, D=2048, dtype="f32", out="bf16", scale=45.25),
        # one more micro-batch into a gradient that is kept in 32 bits, odd sizes
        dict(name="embed_grad_add", op="embed_grad", T=1001, N=50257, D=1537, dtype="bf16", out="f32", scale=1.0, add=True, one=0.0),
        # a training batch's gradient, written whole; a quarter of the tokens is padding by one token
        dict(name="embed_grad_train", op="embed_grad", T=16384, N=128256, D=4096, dtype="bf16", out="bf16", scale=1.0, add=False, one=0.25),
        # the gradients of a tiny drafter
        dict(name="clip_small", op="clip", layers=2, width=256, V=1024, dtype="f32", most=1.0),
        # the gradients of a drafter of half a billion parameters, norms' gains in 32 bits
        dict(name="clip_large", op="clip", layers=24, width=1024, V=128256, dtype="bf16", most=1.0),
    ]


def _between(rng, low, high):
    """A whole number whose logarithm is spread evenly over the range."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["scores", "scores", "scores_grad", "scores_grad", "embed", "embed_grad", "clip"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("scores", "scores_grad"):
        V = rng.choice([32000, 50257, 128256, 152064, _between(rng, 1000, 152064)])
        most = 1024 if op == "scores" else 2048
        case = dict(op=op, R=_between(rng, 1, min(most, MOST_ENTRIES * 3 // 4 // V)), V=V, G=rng.randint(1, 17), dtype=dtype,
                    temp=rng.choice([1.0, rng.uniform(0.5, 1.5)]), pad=rng.choice([0, rng.randint(1, 64)]))
        if op == "scores":
            case.update(M=_between(rng, 1, 128), masked=rng.choice([0.0, 0.0, rng.uniform(0.1, 0.9)]))
        else:
            case["entropy"] = rng.choice([False, True])
        return case
    if op == "clip":
        width = _between(rng, 64, 1024)
        V = _between(rng, 1000, 128256)
        layers = rng.randint(1, 24)
        return dict(op=op, layers=layers, width=width, V=V, dtype=dtype if dtype == "bf16" or layers * width <= 12288 else "bf16",
                    most=rng.choice([1.0, 0.25, 1e6]))
    D = _between(rng, 64, 4096)
    N = _between(rng, 1000, min(128256, MOST_TABLE // D))
    case = dict(op=op, T=_between(rng, 1, MOST_TOKENS), N=N, D=D, dtype=dtype, out=rng.choice(["f32", "bf16"]), scale=rng.choice([1.0, math.sqrt(D)]))
    if op == "embed_grad":
        case.update(add=rng.choice([False, True]), one=rng.choice([0.0, 0.0, rng.uniform(0.05, 0.5)]))
        if D * N > MOST_TABLE // 2:
            case["dtype"] = case["out"] = "bf16"
    return case


# ---- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _logits(R, V, dtype, masked, pad, g):
    """Zipf-like rows with noise, some entries ruled out; `pad` more columns in the buffer behind every row."""
    x = torch.rand(R, V + pad, generator=g, device=DEV)
    x = torch.log_(x.mul_(V).floor_().add_(1.0)).mul_(-1.1).add_(torch.randn(R, V + pad, generator=g, device=DEV), alpha=0.5)
    if masked > 0:
        x.masked_fill_(torch.rand(R, V + pad, generator=g, device=DEV) < masked, -math.inf)
    return x.to(TYPES[dtype])[:, :V]


def _drawn(x, G, temp, g):
    """G tokens a row drawn from its distribution; a few slots hold none, as where a block ended early."""
    t = torch.multinomial(torch.softmax(x.float() / temp, dim=1), G, replacement=True, generator=g)
    none = torch.rand(t.shape, generator=g, device=DEV) < (0.05 if G > 1 else 0.0)
    return torch.where(none, -1, t).to(torch.int32)


def _text(T, N, one, g):
    """Token ids as in text: frequent ones over and over, and a share `one` that is all the same token."""
    t = (torch.rand(T, generator=g, device=DEV).mul(math.log(N)).exp() - 1.0).long().clamp_(0, N - 1)
    t = (t * 7919 + 13) % N
    return torch.where(torch.rand(T, generator=g, device=DEV) < one, 0, t).to(torch.int32)


def _shapes(layers, width, V):
    layer = [(width, width)] * 4 + [(4 * width, width)] * 2 + [(width, 4 * width)] + [(width,)] * 2
    return [(V, width)] + layer * layers + [(width,), (7, width)]


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    state = {"case": case}
    if op in ("scores", "scores_grad"):
        x = _logits(case["R"], case["V"], case["dtype"], case.get("masked", 0.0), case["pad"], g)
        state["x"] = x
        state["tokens"] = _drawn(x, case["G"], case["temp"], g)
        if op == "scores_grad":
            state["a"] = torch.randn(case["R"], case["G"], generator=g, device=DEV) / case["R"]
            state["b"] = torch.full((case["R"],), 0.01 / case["R"], device=DEV) if case["entropy"] else None
    elif op == "embed":
        state["table"] = torch.randn(case["N"], case["D"], generator=g, device=DEV).mul_(0.02).to(TYPES[case["dtype"]])
        state["tokens"] = _text(case["T"], case["N"], 0.0, g)
    elif op == "embed_grad":
        state["g"] = torch.randn(case["T"], case["D"], generator=g, device=DEV).to(TYPES[case["dtype"]])
        state["tokens"] = _text(case["T"], case["N"], case["one"], g)
        if case["add"]:  # (what the earlier micro-batches left; a pass adds to it in place)
            state["sum"] = torch.randn(case["N"], case["D"], generator=g, device=DEV).to(TYPES[case["out"]])
    else:
        shapes = _shapes(case["layers"], case["width"], case["V"])
        state["grads"] = [torch.randn(s, generator=g, device=DEV).mul_(0.01).to(TYPES[case["dtype"]] if len(s) > 1 else torch.float32)
                          for s in shapes]
        # the optimiser's flat buffers, one of matrices and one of gains, which the clipped gradients go to
        state["flat"] = [torch.empty(sum(t.numel() for t in state["grads"] if (t.dim() > 1) == matrices), device=DEV,
                                     dtype=TYPES[case["dtype"]] if matrices else torch.float32) for matrices in (True, False)]
        views = [iter(flat.split([t.numel() for t in state["grads"] if (t.dim() > 1) == matrices]))
                 for flat, matrices in zip(state["flat"], (True, False))]
        state["clipped"] = [next(views[0] if t.dim() > 1 else views[1]).view(t.shape) for t in state["grads"]]
    return state


# ---- plain forms

def _plain_rows(x, temp):
    y = x.float() / temp
    y = torch.where(torch.isfinite(y), y, -math.inf)
    y = y - y.amax(dim=1, keepdim=True)
    lp = y - y.exp().sum(dim=1, keepdim=True).log()
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
    return lp, p, entropy


def _plain_picked(lp, tokens):
    at = tokens.long()
    return torch.where(at >= 0, lp.gather(1, at.clamp(min=0)), 0.0)


def _plain_scores(x, tokens, M, temp):
    lp, _, entropy = _plain_rows(x, temp)
    # the order of the values and, where they are equal, of the indexes, as one whole number
    bits = (x.float() + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(1 << 31) - bits, bits)
    key = bits * (1 << 32) + torch.arange(x.shape[1] - 1, -1, -1, device=x.device)
    ids = x.shape[1] - 1 - (key.topk(M, dim=1).values & 0xFFFFFFFF)
    top = lp.gather(1, ids)
    return {"logp": _plain_picked(lp, tokens), "entropy": entropy,
            "top_ids": torch.where(torch.isfinite(top), ids, -1).to(torch.int32), "top_logp": top}


def _plain_scores_grad(x, tokens, a, b, temp):
    lp, p, entropy = _plain_rows(x, temp)
    valid = tokens >= 0
    a_in = torch.where(valid, a, 0.0)
    back = a_in.sum(dim=1, keepdim=True).expand_as(p)
    if b is not None:
        back = back + b[:, None] * (torch.where(p > 0, lp, 0.0) + entropy[:, None])
    d = (-p * back).scatter_add(1, tokens.long().clamp(min=0), a_in)
    return {"grad": (d / temp).to(x.dtype), "logp": _plain_picked(lp, tokens), "entropy": entropy}


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2506_05632_amd as llc
        if op == "scores":
            return llc.llc_token_logprobs(state["x"], state["tokens"], case["M"], temp=case["temp"])
        if op == "scores_grad":
            return llc.llc_token_logprobs_grad(state["x"], state["tokens"], state["a"], grad_entropy=state["b"], temp=case["temp"])
        if op == "embed":
            return llc.llc_embed(state["table"], state["tokens"], scale=case["scale"], out_dtype=TYPES[case["out"]])
        if op == "embed_grad":
            if case["add"]:
                return llc.llc_embed_grad(state["g"], state["tokens"], case["N"], scale=case["scale"], out=state["sum"], add=True)
            return llc.llc_embed_grad(state["g"], state["tokens"], case["N"], scale=case["scale"], out_dtype=TYPES[case["out"]])
        found = llc.llc_clip_grad_norm(state["grads"], case["most"], out=state["clipped"])
        return {"norm": found["norm"], "clipped": state["flat"]}
    if op == "scores":
        return _plain_scores(state["x"], state["tokens"], case["M"], case["temp"])
    if op == "scores_grad":
        return _plain_scores_grad(state["x"], state["tokens"], state["a"], state["b"], case["temp"])
    if op == "embed":
        return {"out": (state["table"][state["tokens"].long()].float() * case["scale"]).to(TYPES[case["out"]])}
    if op == "embed_grad":
        total = state["sum"].float() if case["add"] else torch.zeros(case["N"], case["D"], device=DEV)  # (float(): itself where it is in 32 bits)
        total.index_add_(0, state["tokens"].long(), state["g"].float() * case["scale"])
        return {"grad": state["sum"].copy_(total) if case["add"] else total.to(TYPES[case["out"]])}
    norm = torch.stack([t.float().square().sum() for t in state["grads"]]).sum().sqrt()
    factor = (case["most"] / norm).clamp(max=1.0)
    state["clipped"] = [c.copy_(t.float() * factor) for c, t in zip(state["clipped"], state["grads"])]
    return {"norm": norm, "clipped": state["flat"]}


# ---- what a pass cannot do without

def work(case):
    size = {"f32": 4, "bf16": 2}
    op, e = case["op"], size[case["dtype"]]
    if op in ("scores", "scores_grad"):
        entries, slots = case["R"] * case["V"], case["R"] * case["G"]
        if op == "scores":  # difference, product, exponential, two sums, one comparison an entry
            return {"bytes": entries * e + slots * 8 + case["R"] * (4 + 8 * case["M"]), "flops": entries * 7}
        return {"bytes": 2 * entries * e + slots * 12 + case["R"] * 8, "flops": entries * 10}
    if op == "embed":
        return {"bytes": case["T"] * (4 + case["D"] * (e + size[case["out"]])), "flops": case["T"] * case["D"]}
    if op == "embed_grad":
        rows = case["N"]
        if case["add"]:  # the rows of the tokens that occur, as many as may be expected, are read and written
            times = torch.log1p(1.0 / torch.arange(1, case["N"] + 1, dtype=torch.float64)) / math.log(case["N"])
            rows = 2 * int((1.0 - (1.0 - times).pow(case["T"] * (1.0 - case["one"]))).sum())
        return {"bytes": case["T"] * (4 + case["D"] * e) + rows * case["D"] * size[case["out"]], "flops": case["T"] * case["D"]}
    shapes = _shapes(case["layers"], case["width"], case["V"])
    return {"bytes": sum(2 * math.prod(s) * (e if len(s) > 1 else 4) for s in shapes), "flops": sum(3 * math.prod(s) for s in shapes)}


# ---- definitions in 64 bits

def _exact_row(x, temp):
    """Log probabilities, entropy and order of some rows, from the sums of exponentials themselves."""
    z = x.double() / float(torch.tensor(temp, dtype=torch.float32))
    lp = z - torch.logsumexp(z, dim=1, keepdim=True)
    return lp, torch.special.entr(lp.exp()).sum(dim=1)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("scores", "scores_grad"):
        parts = []
        step = max(1, (1 << 24) // case["V"])
        for r in range(0, case["R"], step):
            x, tokens = state["x"][r:r + step], state["tokens"][r:r + step].long()
            lp, entropy = _exact_row(x, case["temp"])
            picked = torch.take_along_dim(lp, tokens.clamp(min=0), dim=1)
            picked[tokens < 0] = 0.0
            if op == "scores":
                order = torch.sort(x.double(), dim=1, descending=True, stable=True)
                ids = order.indices[:, :case["M"]].clone()
                ids[torch.isinf(order.values[:, :case["M"]])] = -1
                parts.append({"logp": picked, "entropy": entropy, "top_ids": ids.to(torch.int32),
                              "top_logp": torch.take_along_dim(lp, order.indices[:, :case["M"]], dim=1)})
                continue
            a = state["a"][r:r + step].double() * (tokens >= 0)
            p = lp.exp()
            d = -p * a.sum(dim=1, keepdim=True)
            if case["entropy"]:
                d -= state["b"][r:r + step, None].double() * p * (lp + entropy[:, None])
            rows = torch.arange(x.shape[0], device=DEV)
            for n in range(case["G"]):
                d[rows, tokens[:, n].clamp(min=0)] += a[:, n]
            d /= float(torch.tensor(case["temp"], dtype=torch.float32))
            parts.append({"grad": d, "logp": picked, "entropy": entropy})
        return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
    if op == "embed":
        return {"out": state["table"].double().index_select(0, state["tokens"].long()) * _single(case["scale"])}
    if op == "embed_grad":
        total = state["sum"].double() if case["add"] else torch.zeros(case["N"], case["D"], dtype=torch.float64, device=DEV)
        order = torch.argsort(state["tokens"].long())
        rows = state["tokens"].long()[order]
        return {"grad": total.index_put_((rows,), state["g"][order].double() * _single(case["scale"]), accumulate=True)}
    norm = math.sqrt(math.fsum(float(t.double().pow(2).sum()) for t in state["grads"]))
    return {"norm": torch.tensor(norm, dtype=torch.float64, device=DEV),
            "clipped": [torch.cat([t.double().reshape(-1) * min(1.0, case["most"] / norm) for t in state["grads"] if (t.dim() > 1) == matrices])
                        for matrices in (True, False)]}


def _single(value):
    return float(torch.tensor(value, dtype=torch.float32))
