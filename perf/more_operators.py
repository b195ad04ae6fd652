"""What is measured of the operators of a drafting step's end: their cases, inputs, plain forms and definitions.

A program that drafts multiplies hidden states with the output layer, cuts the distribution to what the request allows
(the likeliest k, a share of the mass, a share of the largest probability) and samples, or hands the cut rows to the
coupling, then looks the tokens up for the next position.  The layer and the table are held in 4 bits with scales of
groups; fitting with such weights rounds them and reads them back in every step.

`run` computes an operator in its plain form, elementary torch operations in 32 bits (64 where a border is decided:
cumulated masses, quotients to be rounded), or, where `own` is true, by the library's call.  `exact` evaluates its definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
MOST_ENTRIES = 1024 * 128256    # logits of the largest listed call
MOST_WEIGHTS = 128256 * 4096    # weights of the largest listed layer
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one serving step of a lightly loaded server: four requests with the usual cuts
        dict(name="sample_step", op="sample", R=4, V=32000, S=1, dtype="bf16", cuts="all", temp=0.8, top_k=40, top_p=0.95, min_p=0.0, pad=0),
        # a full batch of requests that each bring their own settings: greedy ones, uncut ones, all kinds of cuts
        dict(name="sample_requests", op="sample", R=256, V=128256, S=1, dtype="bf16", cuts="rows", pad=0),
        # eight drafts of every row from a share of the mass, on a large vocabulary
        dict(name="sample_nucleus", op="sample", R=1024, V=128256, S=8, dtype="f32", cuts="all", temp=0.7, top_k=0, top_p=0.9, min_p=0.0, pad=0),
        # an odd vocabulary, rows of a wider buffer, cut before the coupling of dense rows
        dict(name="truncate_odd", op="truncate", R=300, V=50257, dtype="f32", cuts="all", temp=0.8, top_k=0, top_p=1.0, min_p=0.05, pad=31),
        # both cuts on the rows of a whole batch, as the couplings read them
        dict(name="truncate_large", op="truncate", R=1024, V=128256, dtype="bf16", cuts="all", temp=1.0, top_k=1000, top_p=0.95, min_p=0.0, pad=0),
        # one projection inside a small drafter, one sequence: the smallest call, latency counts
        dict(name="matvec_step", op="matvec", R=1, N=2048, D=2048, G=128, dtype="bf16", scales="bf16", out="bf16", zeros=False),
        # the output layer on a large vocabulary for the drafts of one request
        dict(name="matvec_head", op="matvec", R=8, N=128256, D=4096, G=128, dtype="bf16", scales="bf16", out="f32", zeros=False),
        # the same layer's kind for a batch of sequences in 32 bits, odd sizes, zeros beside the scales
        dict(name="matvec_batch", op="matvec", R=61, N=50257, D=2050, G=64, dtype="f32", scales="f32", out="f32", zeros=True),
        # fitting with rounded weights: an output layer's master copy to 4 bits and back
        dict(name="quantize_fit", op="quantize", N=128256, D=2048, G=64, dtype="f32", scales="bf16", out="bf16", zeros=True),
        # a small layer of odd sizes, small groups
        dict(name="quantize_odd", op="quantize", N=2000, D=1537, G=32, dtype="bf16", scales="f32", out="f32", zeros=False),
        # the lookup of one drafting step: eight requests with four drafts each
        dict(name="embed_step", op="embed", T=32, N=32000, D=2048, G=128, scales="bf16", out="bf16", zeros=False, scale=1.0),
        # the lookup of a long prompt, scaled by the root of the width
        dict(name="embed_prompt", op="embed", T=16384, N=128256, D=4096, G=64, scales="bf16", out="bf16", zeros=True, scale=64.0),
    ]


def _between(rng, low, high):
    """A whole number whose logarithm is spread evenly over the range."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "truncate", "matvec", "matvec", "quantize", "embed"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("sample", "truncate"):
        V = rng.choice([32000, 50257, 128256, 152064, _between(rng, 1000, 152064)])
        case = dict(op=op, R=_between(rng, 1, min(1024, MOST_ENTRIES * 3 // 4 // V)), V=V, dtype=dtype, cuts=rng.choice(["all", "all", "rows"]),
                    pad=rng.choice([0, rng.randint(1, 64)]))
        if op == "sample":
            case["S"] = _between(rng, 1, 16)
        if case["cuts"] == "all":
            case.update(temp=rng.choice([1.0, rng.uniform(0.4, 1.5)]), top_k=rng.choice([0, 0, _between(rng, 1, 2000)]),
                        top_p=rng.choice([1.0, rng.uniform(0.5, 0.99)]), min_p=rng.choice([0.0, 0.0, rng.uniform(0.01, 0.2)]))
        return case
    case = dict(op=op, G=rng.choice([32, 64, 128]), scales=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]), zeros=rng.choice([False, True]))
    D = _between(rng, 64, 8192)
    if op == "matvec":
        R = _between(rng, 1, 64)
        case.update(R=R, N=_between(rng, 64, min(152064, MOST_WEIGHTS // 2 // D)), D=D, dtype=dtype)
    elif op == "quantize":
        case.update(N=_between(rng, 64, min(128256, MOST_WEIGHTS // 4 // D)), D=D, dtype=dtype)
    else:
        case.update(T=_between(rng, 1, min(16384, (1 << 25) // D)), N=_between(rng, 1000, min(128256, MOST_WEIGHTS // 2 // D)), D=D,
                    scale=rng.choice([1.0, math.sqrt(D)]))
    return case


# ---- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _logits(R, V, dtype, pad, g):
    """Zipf-like rows with noise, from nearly flat to sharply peaked ones as a model's next tokens are; `pad` more columns behind every row."""
    x = torch.rand(R, V + pad, generator=g, device=DEV)
    steep = 1.1 + 2.4 * torch.rand(R, 1, generator=g, device=DEV)
    return torch.log_(x.mul_(V).floor_().add_(1.0)).mul_(-steep).add_(torch.randn(R, V + pad, generator=g, device=DEV), alpha=0.5).to(TYPES[dtype])[:, :V]


def _settings(case, g):
    """Temperature and cuts: one set for all rows, or each row's own as requests bring them."""
    if case["cuts"] == "all":
        return {name: case[name] for name in ("temp", "top_k", "top_p", "min_p")}
    R = case["R"]
    what = torch.rand(4, R, generator=g, device=DEV)
    value = torch.rand(4, R, generator=g, device=DEV)
    top_k = torch.where(what[1] < 0.15, 1, torch.where(what[1] < 0.6, (10 + 90 * value[1]).long(), 0))
    return {"temp": torch.where(what[0] < 0.4, 1.0, 0.4 + 0.8 * value[0]), "top_k": top_k.to(torch.int32),
            "top_p": torch.where(what[2] < 0.4, 1.0, 0.6 + 0.39 * value[2]), "min_p": torch.where(what[3] < 0.7, 0.0, 0.02 + 0.1 * value[3])}


def _text(T, N, g):
    """Token ids as in text: frequent ones over and over; a few slots hold none."""
    t = (torch.rand(T, generator=g, device=DEV).mul(math.log(N)).exp() - 1.0).long().clamp_(0, N - 1)
    t = (t * 7919 + 13) % N
    return torch.where(torch.rand(T, generator=g, device=DEV) < 0.02, -1, t).to(torch.int32)


def _layer(case, g):
    """A layer as a program keeps it: two entries a byte, a scale (and a zero) of every group."""
    N, D, groups = case["N"], case["D"], -(-case["D"] // case["G"])
    codes = torch.empty(N, (D + 1) // 2, dtype=torch.uint8, device=DEV)
    for n in range(0, N, 16384):
        part = codes[n:n + 16384]
        q = torch.randn(2, *part.shape, generator=g, device=DEV).mul_(2.5).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
        part.copy_(q[0] | (q[1] << 4))
    state = {"codes": codes, "scales": (0.004 + 0.004 * torch.rand(N, groups, generator=g, device=DEV)).to(TYPES[case["scales"]]), "zeros": None}
    if case["zeros"]:
        state["zeros"] = torch.randint(5, 11, (N, groups), generator=g, device=DEV, dtype=torch.uint8)
    return state


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op in ("sample", "truncate"):
        state = {"x": _logits(case["R"], case["V"], case["dtype"], case["pad"], g), "settings": _settings(case, g)}
        if op == "sample":
            state["u"] = torch.rand(case["R"], case["S"], generator=g, device=DEV)
    elif op == "quantize":
        # channels of different size, as a layer's rows have
        state = {"w": (torch.randn(case["N"], case["D"], generator=g, device=DEV)
                       * (0.01 + 0.02 * torch.rand(case["N"], 1, generator=g, device=DEV))).to(TYPES[case["dtype"]]),
                 "rows": torch.arange(case["N"], dtype=torch.int32, device=DEV)}
    else:
        state = _layer(case, g)
        if op == "matvec":
            # hidden states with a few channels far larger than the others
            large = 1.0 + 20.0 * (torch.rand(case["D"], generator=g, device=DEV) < 0.01)
            state["x"] = (torch.randn(case["R"], case["D"], generator=g, device=DEV) * large).to(TYPES[case["dtype"]])
        else:
            state["tokens"] = _text(case["T"], case["N"], g)
    state["case"] = case
    return state


# ---- plain forms

def _column(value, like, dtype):
    return (value if isinstance(value, torch.Tensor) else torch.tensor(value, dtype=torch.float32, device=like.device).expand(like.shape[0])).to(dtype)[:, None]


def _plain_kept(x, settings):
    """What the cuts leave of every row: which entries, and all entries' masses relative to the largest."""
    V = x.shape[1]
    bits = (x.float() + 0.0).view(torch.int32).long()  # the order of the values and, where they are equal, of the indexes, as one whole number
    bits = torch.where(bits < 0, -(1 << 31) - bits, bits)
    order = (bits * (1 << 32) + torch.arange(V - 1, -1, -1, device=x.device)).argsort(dim=1, descending=True)
    z = x.double()
    z = (z - z.amax(dim=1, keepdim=True)) / _column(settings["temp"], x, torch.float64)
    sorted_z = z.gather(1, order)
    mass = sorted_z.exp()
    rank = torch.arange(V, device=x.device)[None, :]
    top_k = _column(settings["top_k"], x, torch.int64)
    keep = (rank < top_k) | (top_k <= 0)
    cumulated = mass.cumsum(dim=1)
    total = torch.where(keep, mass, 0.0).sum(dim=1, keepdim=True)
    top_p = _column(settings["top_p"], x, torch.float64)
    keep &= (cumulated - mass < top_p * total) | (top_p >= 1.0)
    keep &= (sorted_z >= _column(settings["min_p"], x, torch.float64).log()) | (rank == 0)
    return torch.zeros_like(keep).scatter(1, order, keep), z


def _plain_sample(x, u, settings):
    kept, z = _plain_kept(x, settings)
    upto = torch.where(kept, z.exp(), 0.0).cumsum(dim=1)
    tokens = torch.searchsorted(upto, u.double() * upto[:, -1:], right=True)
    return {"tokens": tokens.to(torch.int32), "logp": (z.gather(1, tokens) - upto[:, -1:].log()).float(), "kept": kept.sum(dim=1).to(torch.int32)}


def _plain_truncate(x, settings):
    kept, _ = _plain_kept(x, settings)
    return {"logits": torch.where(kept, x, -math.inf), "kept": kept.sum(dim=1).to(torch.int32)}


def _plain_values(codes, scales, zeros, D, G):
    q = torch.stack([codes & 15, codes >> 4], dim=2).flatten(1)[:, :D].float()
    at = torch.arange(D, device=codes.device) // G
    zero = 8.0 if zeros is None else zeros.float().index_select(1, at)
    return (q - zero) * scales.float().index_select(1, at)


def _plain_quantize(w, G, scales, zeros, out):
    N, D = w.shape
    groups = -(-D // G)
    padded = torch.zeros(N, groups * G, device=w.device)
    padded[:, :D] = w
    v = padded.view(N, groups, G)
    if zeros:
        low, high = v.amin(dim=2).clamp(max=0.0), v.amax(dim=2).clamp(min=0.0)
        scale = ((high - low).double() / 15.0).float().to(scales)
        zero = torch.where(scale > 0, (-low.double() / scale.double()).round().clamp(0, 15), 8.0).float()
    else:
        scale = (v.abs().amax(dim=2).double() / 7.0).float().to(scales)
        zero = torch.full_like(scale, 8.0, dtype=torch.float32)
    s = scale.float()[:, :, None]
    q = torch.where(s > 0, (v.double() / s.double()).round() + zero[:, :, None], zero[:, :, None]).clamp(0, 15).float()  # (32 bits make ties of quotients that are none)
    values = ((q - zero[:, :, None]) * s).view(N, -1)[:, :D].to(out)
    return {"values": values, "scales": scale, "zeros": zero.to(torch.uint8) if zeros else None}


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2506_05632_amd as llc
        if op == "sample":
            return llc.llc_sample(state["x"], state["u"], want_kept=True, **state["settings"])
        if op == "truncate":
            return llc.llc_truncate(state["x"], **state["settings"])
        if op == "matvec":
            return llc.llc_matvec_quantized(state["x"], state["codes"], state["scales"], zeros=state["zeros"], group=case["G"], out_dtype=TYPES[case["out"]])
        if op == "embed":
            return llc.llc_embed_quantized(state["codes"], state["scales"], state["tokens"], case["D"], zeros=state["zeros"], group=case["G"],
                                  scale=case["scale"], out_dtype=TYPES[case["out"]])
        q = llc.llc_quantize(state["w"], group=case["G"], zeros=case["zeros"], scales_dtype=TYPES[case["scales"]])
        back = llc.llc_embed_quantized(q["codes"], q["scales"], state["rows"], case["D"], zeros=q.get("zeros"), group=case["G"], out_dtype=TYPES[case["out"]])
        return {"values": back["out"], "scales": q["scales"], "zeros": q.get("zeros")}
    if op == "sample":
        return _plain_sample(state["x"], state["u"], state["settings"])
    if op == "truncate":
        return _plain_truncate(state["x"], state["settings"])
    if op == "matvec":
        w = _plain_values(state["codes"], state["scales"], state["zeros"], case["D"], case["G"])
        return {"out": (state["x"].float() @ w.t()).to(TYPES[case["out"]])}
    if op == "embed":
        at = state["tokens"].long().clamp(min=0)
        w = _plain_values(state["codes"][at], state["scales"][at], None if state["zeros"] is None else state["zeros"][at], case["D"], case["G"])
        return {"out": torch.where(state["tokens"][:, None] >= 0, w * case["scale"], 0.0).to(TYPES[case["out"]])}
    return _plain_quantize(state["w"], case["G"], TYPES[case["scales"]], case["zeros"], TYPES[case["out"]])


# ---- what a pass cannot do without

def work(case):
    op = case["op"]
    if op in ("sample", "truncate"):
        entries = case["R"] * case["V"]
        rows = case["R"] * (0 if case["cuts"] == "all" else 16)  # the rows' settings
        more = case["R"] * (4 + 12 * case["S"]) if op == "sample" else case["R"] * 4 + entries * SIZE[case["dtype"]]
        return {"bytes": entries * SIZE[case["dtype"]] + rows + more, "flops": entries * 5}  # difference, product, exponential, sum, comparison
    groups = -(-case["D"] // case["G"])
    row = (case["D"] + 1) // 2 + groups * (SIZE[case["scales"]] + (1 if case["zeros"] else 0))
    if op == "matvec":
        return {"bytes": case["N"] * row + case["R"] * (case["D"] * SIZE[case["dtype"]] + case["N"] * SIZE[case["out"]]),
                "flops": 2 * case["R"] * case["N"] * case["D"]}
    if op == "embed":
        return {"bytes": case["T"] * (4 + row + case["D"] * SIZE[case["out"]]), "flops": 2 * case["T"] * case["D"]}
    entries = case["N"] * case["D"]  # in, to 4 bits, and back
    return {"bytes": entries * (SIZE[case["dtype"]] + SIZE[case["out"]]) + 2 * case["N"] * row, "flops": 6 * entries}


# ---- definitions in 64 bits

def _single(value, R):
    """A setting as every row has it, the number that 32 bits hold."""
    t = value if isinstance(value, torch.Tensor) else torch.full((R,), float(value), device=DEV)
    return t.double()


def _exact_rows(x, temp, top_k, top_p, min_p):
    """Kept entries and probabilities of some rows: the shortest run of the sorted row that meets every cut."""
    R, V = x.shape
    p = torch.softmax(x.double() / temp[:, None], dim=1)
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices
    down = torch.take_along_dim(p, order, dim=1)
    sums = torch.cumsum(down, dim=1)
    count = torch.where(top_k > 0, top_k, float(V)).clamp(max=V).long()
    limit = top_p * torch.take_along_dim(sums, (count - 1)[:, None], dim=1)[:, 0]
    reached = torch.searchsorted(sums, limit[:, None])[:, 0] + 1
    count = torch.where(top_p < 1.0, torch.minimum(count, reached), count)
    likely = torch.log(down) - torch.log(down[:, :1])
    count = torch.minimum(count, (likely >= torch.log(min_p)[:, None] - 1e-13).sum(dim=1).clamp(min=1))
    places = torch.empty_like(order)
    places.scatter_(1, order, torch.arange(V, device=DEV).expand(R, V))
    return places < count[:, None], p, count


def _exact_cut(case, state):
    R, V = case["R"], case["V"]
    settings = [_single(state["settings"][name], R) for name in ("temp", "top_k", "top_p", "min_p")]
    parts = []
    step = max(1, (1 << 25) // V)
    for r in range(0, R, step):
        x = state["x"][r:r + step]
        kept, p, count = _exact_rows(x, *(s[r:r + step] for s in settings))
        part = {"kept": count.to(torch.int32)}
        if case["op"] == "truncate":
            part["logits"] = x.double().masked_fill(~kept, -math.inf)
        else:
            inside = p * kept
            sums = inside.cumsum(dim=1)
            total = sums[:, -1:]
            at = (sums[:, None, :] <= (state["u"][r:r + step].double() * total)[:, :, None]).sum(dim=2) if V * sums.shape[0] * case["S"] < 1 << 27 else \
                torch.stack([(sums <= state["u"][r:r + step, s:s + 1].double() * total).sum(dim=1) for s in range(case["S"])], dim=1)
            part["tokens"] = at.to(torch.int32)
            part["logp"] = torch.log(inside.gather(1, at) / total)
        parts.append(part)
    names = ("tokens", "logp", "kept") if case["op"] == "sample" else ("logits", "kept")
    return {name: torch.cat([p[name] for p in parts]) for name in names}


def _exact_values(codes, scales, zeros, D, G):
    q = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=DEV)
    q[:, 0::2] = codes.remainder(16)
    q[:, 1::2] = codes.div(16, rounding_mode="floor")
    spread = lambda t: t.double().repeat_interleave(G, dim=1)[:, :D]  # noqa: E731
    return (q[:, :D] - (8 if zeros is None else spread(zeros))) * spread(scales)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("sample", "truncate"):
        return _exact_cut(case, state)
    if op == "embed":
        out = torch.zeros(case["T"], case["D"], dtype=torch.float64, device=DEV)
        held = state["tokens"] >= 0
        at = state["tokens"][held].long()
        out[held] = _exact_values(state["codes"][at], state["scales"][at], None if state["zeros"] is None else state["zeros"][at],
                                  case["D"], case["G"]) * float(torch.tensor(case["scale"], dtype=torch.float32))
        return {"out": out}
    if op == "matvec":
        x, parts = state["x"].double(), []
        for n in range(0, case["N"], 8192):
            zeros = None if state["zeros"] is None else state["zeros"][n:n + 8192]
            parts.append(torch.mm(x, _exact_values(state["codes"][n:n + 8192], state["scales"][n:n + 8192], zeros, case["D"], case["G"]).t().contiguous()))
        return {"out": torch.cat(parts, dim=1)}
    N, D, G = case["N"], case["D"], case["G"]
    values, scales, zeros = [], [], []
    for first in range(0, D, G):
        v = state["w"][:, first:first + G].double()
        if case["zeros"]:
            low, high = v.amin(dim=1).clamp(max=0.0), v.amax(dim=1).clamp(min=0.0)
            s = ((high.float() - low.float()).double() / 15.0).to(TYPES[case["scales"]])
            zero = torch.round(-low / s.double()).clamp(0, 15)
        else:
            s = (v.abs().amax(dim=1) / 7.0).to(TYPES[case["scales"]])
            zero = torch.full((N,), 8.0, dtype=torch.float64, device=DEV)
        q = (torch.round(v / s.double()[:, None]) + zero[:, None]).clamp(0, 15)
        values.append((q - zero[:, None]) * s.double()[:, None])
        scales.append(s.double())
        zeros.append(zero.to(torch.uint8))
    return {"values": torch.cat(values, dim=1), "scales": torch.stack(scales, dim=1), "zeros": torch.stack(zeros, dim=1) if case["zeros"] else None}
