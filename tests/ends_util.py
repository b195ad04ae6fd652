"""Plain 64-bit evaluations of the operators at the vocabulary's two ends, on the host, and the tolerances they are held to.

What the kernels round: a row's sums are formed in fp32 by threads that add at most a few hundred terms each (a relative
2^-24 an addition, random in sign, and as much for the exponential), so that ln of the sum is within 2e-6; the exponent of a term
at distance d from the largest is within 2^-23 d; outputs are rounded once."""
import numpy as np
import torch

SUM = 2e-6       # ln of a row's sum
STEP = 2.0 ** -23  # an exponent, for each unit of distance; an fp32 output, relative
OUT = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}  # an output's rounding, relative


def rows(x, temp):
    """x [R,V] (any float tensor) -> (the largest x, 0 without mass, and ln sum exp((x - largest) / temp)) [R,2], p, ln p, entropy.

    (ln p is taken from those two parts: their sum loses the second where the values are large.)"""
    y = x.detach().cpu().double().numpy()
    y = np.where(np.isfinite(y), y, -np.inf)
    top = y.max(axis=1, keepdims=True)
    any_mass = np.isfinite(top)
    top = np.where(any_mass, top, 0.0)
    y = (y - top) / np.float64(np.float32(temp))
    e = np.exp(y)
    with np.errstate(divide="ignore", invalid="ignore"):
        rest = np.log(e.sum(axis=1, keepdims=True))
        lp = np.where(np.isfinite(y), y - rest, -np.inf)
        p = np.exp(lp)
        entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(axis=1)
    return np.concatenate([top, rest], axis=1), p, lp, entropy


def scores(x, tokens, M, temp):
    V = x.shape[1]
    lse, _, lp, entropy = rows(x, temp)
    t = tokens.cpu().numpy().reshape(x.shape[0], -1).astype(np.int64) if tokens is not None else np.zeros((x.shape[0], 0), np.int64)
    logp = np.take_along_axis(lp, np.clip(t, 0, V - 1), axis=1)
    logp = np.where(t < 0, 0.0, np.where(t >= V, -np.inf, logp))
    v = x.detach().cpu().double().numpy()
    v = np.where(np.isfinite(v), v, -np.inf)
    order = np.argsort(-v, axis=1, kind="stable")[:, :M]
    top = np.take_along_axis(lp, order, axis=1)
    ids = np.where(np.isfinite(np.take_along_axis(v, order, axis=1)), order, -1)
    fill = M - ids.shape[1]
    ids = np.pad(ids, ((0, 0), (0, max(fill, 0))), constant_values=-1)
    top = np.pad(top, ((0, 0), (0, max(fill, 0))), constant_values=-np.inf)
    return {"logp": logp, "entropy": entropy, "lse": lse, "top_ids": ids, "top_logp": top}


def close(got, want, atol, rtol):
    """Equal where not finite (in the output's type), near elsewhere."""
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64) if got.dtype == torch.float32 else want
    got = got.detach().cpu().double().numpy().reshape(want.shape)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine])
    got, want = got[fine], want[fine]
    far = np.abs(got - want) - (atol + rtol * np.abs(want))
    assert far.size == 0 or far.max() <= 0, (far.max(), got[far.argmax()], want[far.argmax()])


def check_scores(out, x, tokens, M, temp):
    want = scores(x, tokens, M, temp)
    if tokens is not None:
        close(out["logp"], want["logp"], SUM, 2 * STEP)
    if "entropy" in out:
        close(out["entropy"], want["entropy"], 2 * SUM, 2 * SUM)
    if "lse" in out:
        close(out["lse"], want["lse"], SUM, 1e-15)
    if M > 0:
        np.testing.assert_array_equal(out["top_ids"].cpu().numpy(), want["top_ids"])
        close(out["top_logp"], want["top_logp"], SUM, 2 * STEP)


def gradient(x, tokens, a, b, temp):
    """The gradient, and the tolerance it is held to, both [R,V]."""
    R, V = x.shape
    _, p, lp, entropy = rows(x, temp)
    T = np.float64(np.float32(temp))
    t = tokens.cpu().numpy().reshape(R, -1).astype(np.int64)
    a = np.where((t >= 0) & (t < V), a.cpu().double().numpy().reshape(R, -1), 0.0)
    b = b.cpu().double().numpy()[:, None] if b is not None else np.zeros((R, 1))
    hot, hot_size = np.zeros((R, V)), np.zeros((R, V))
    for r in range(R):
        np.add.at(hot[r], np.clip(t[r], 0, V - 1), a[r])
        np.add.at(hot_size[r], np.clip(t[r], 0, V - 1), np.abs(a[r]))
    far = np.where(p > 0, np.abs(np.where(p > 0, lp, 0.0)), 0.0)
    d = (hot - p * (a.sum(axis=1, keepdims=True) + b * np.where(p > 0, np.where(p > 0, lp, 0.0) + entropy[:, None], 0.0))) / T
    mass = np.isfinite(x.detach().cpu().double().numpy())
    d = np.where(mass, d, 0.0)
    weight = p * (np.abs(a).sum(axis=1, keepdims=True) + np.abs(b) * (far + entropy[:, None] + 1.0))
    tol = (weight * (4 * SUM + 4 * STEP * far) + hot_size * 4 * STEP * a.shape[1]) / T
    return d, np.where(mass, tol, 0.0) + OUT[x.dtype] * np.abs(d) + 2.0 ** -126
