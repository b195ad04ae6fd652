"""Plain 64-bit evaluations of the operators at a drafting step's end, on the host."""
import bisect
import math
from fractions import Fraction

import numpy as np
import torch

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step, relative


def _rows(value, R):
    if isinstance(value, torch.Tensor):
        return value.detach().cpu().double().numpy()
    return np.full(R, np.float64(np.float32(value)))


def _sums(masses):
    """Running sums of masses in [0, 1], exact to 2^-90 a term, as whole numbers of 2^-90 (equal masses give equal terms)."""
    total, out = 0, []
    for m in masses:
        total += int(math.ldexp(m, 90))
        out.append(total)
    return out


# Where a border of the sums lies within this share of the whole from what it is compared with, 64 bits cannot tell the sides: a
# sum by tiles takes 8 + 6 + 256 additions at most in a row here, each 2^-53, and the exponentials are within 2^-48.  Histograms
# count units of 2^-52 of the largest mass at most, half a unit off an entry, of 2^17 entries.
SIDE = 2.0 ** -44
SIDE_OF_CUT = 2.0 ** -35


def cut(x, temp=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """x [R,V] -> kept [R,V], masses relative to the largest [R,V], by the definition: a run of the sorted row; and [R], where the share of the mass
    ends the run so near to a border that 64 bits cannot tell on which side of an entry, the other possible length (0: none)."""
    y = x.detach().cpu().double().numpy()
    R, V = y.shape
    y = np.where(np.isfinite(y), y, -np.inf)
    temp, top_k, top_p, min_p = (_rows(v, R) for v in (temp, top_k, top_p, min_p))
    kept, mass, other = np.zeros((R, V), bool), np.zeros((R, V)), np.zeros(R, int)
    for r in range(R):
        n_all = int(np.isfinite(y[r]).sum())
        if n_all == 0 or not (2.0 ** -126 <= temp[r] < np.inf) or np.isnan(top_p[r]) or np.isnan(min_p[r]):
            continue
        order = np.argsort(-y[r], kind="stable")[:n_all]
        z = (y[r][order] - y[r][order[0]]) / temp[r]
        m = np.exp(z)
        n = int(top_k[r]) if 0 < top_k[r] < n_all else n_all
        n_min = max(1, int((z >= math.log(min(min_p[r], 1.0))).sum())) if min_p[r] > 0 else n_all
        if top_p[r] < 1:
            upto = _sums(m)
            part = Fraction(max(float(top_p[r]), 0.0)) * upto[n - 1]
            n_p = bisect.bisect_left(upto, math.ceil(part)) + 1
            if not set(np.unique(m)) <= {0.0, 1.0}:
                if n_p > 1 and part - upto[n_p - 2] < SIDE_OF_CUT * upto[n - 1]:
                    other[r] = min(n_p - 1, n_min)
                elif n_p < n and upto[n_p - 1] - part < SIDE_OF_CUT * upto[n - 1]:
                    other[r] = min(n_p + 1, n_min)
            n = min(n, n_p)
        n = max(1, min(n, n_min))
        if other[r] == n:
            other[r] = 0
        kept[r, order[:n]] = True
        mass[r, order] = m
    return kept, mass, other


def _run(x, r, n):
    """The first n entries of row r in order, of those with mass."""
    y = x[r].detach().cpu().double().numpy()
    kept = np.zeros(len(y), bool)
    kept[np.argsort(-np.where(np.isfinite(y), y, -np.inf), kind="stable")[:n]] = True
    return kept


def _settle(kept, other, x, got):
    """The runs whose length 64 bits cannot tell, as long as the call has them if that is the other possible length."""
    for r in np.nonzero(other)[0]:
        if got[r] == other[r]:
            kept[r] = _run(x, r, other[r])


def check_sample(out, x, u, **settings):
    kept, mass, other = cut(x, **settings)
    _settle(kept, other, x, out["kept"].cpu().numpy())
    np.testing.assert_array_equal(out["kept"].cpu().numpy(), kept.sum(axis=1))
    R = x.shape[0]
    temp = _rows(settings.get("temp", 1.0), R)
    u = u.detach().cpu().double().numpy().reshape(R, -1)
    got, logp = out["tokens"].cpu().numpy().reshape(u.shape), out["logp"].cpu().double().numpy().reshape(u.shape)
    y = x.detach().cpu().double().numpy()
    for r in range(R):
        at = np.nonzero(kept[r])[0]
        if len(at) == 0:
            assert (got[r] == -1).all() and (logp[r] == -np.inf).all()
            continue
        m = mass[r][at]
        upto, exact = _sums(m), set(np.unique(m)) <= {0.0, 1.0}
        top = y[r][at].max()
        for s in range(u.shape[1]):
            if np.isnan(u[r, s]):
                assert got[r, s] == -1 and logp[r, s] == -np.inf
                continue
            target = Fraction(min(max(u[r, s], 0.0), 1.0)) * upto[-1]
            i = min(bisect.bisect_right(upto, math.floor(target)), len(at) - 1)
            if got[r, s] != at[i]:
                j = int(np.searchsorted(at, got[r, s]))
                assert not exact and at[min(j, len(at) - 1)] == got[r, s] and abs(upto[min(i, j)] - target) <= SIDE * upto[-1] and abs(upto[max(i, j) - 1] - target) <= SIDE * upto[-1], (r, s, got[r, s], at[i])
                i = j
            want = (y[r, at[i]] - top) / temp[r] - math.log(math.ldexp(upto[-1], -90))
            # in 64 bits, rounded once; at 0 what 64 bits leave of the difference
            assert abs(logp[r, s] - want) <= 1.01 * 2.0 ** -24 * abs(want) + 1e-12, (r, s, logp[r, s], want)


def check_truncate(out, x, **settings):
    kept, _, other = cut(x, **settings)
    _settle(kept, other, x, out["kept"].cpu().numpy())
    np.testing.assert_array_equal(out["kept"].cpu().numpy(), kept.sum(axis=1))
    want = torch.where(torch.from_numpy(kept), x.detach().cpu(), torch.tensor(-math.inf, dtype=x.dtype))
    assert torch.equal(out["logits"].cpu(), want)


def codes_of(codes, D):
    c = codes.detach().cpu().numpy()
    return np.stack([c & 15, c >> 4], axis=2).reshape(c.shape[0], 2 * c.shape[1])[:, :D].astype(np.float64)


def values(codes, scales, zeros, D, group):
    at = np.arange(D) // group
    zero = 8.0 if zeros is None else zeros.detach().cpu().double().numpy()[:, at]
    return (codes_of(codes, D) - zero) * scales.detach().cpu().double().numpy()[:, at]


def quantize(w, group, zeros, scales_dtype):
    """codes [N,D], scales (of their type), zeros, by the definition: quotients as real numbers."""
    w64 = w.detach().cpu().double().numpy()
    N, D = w64.shape
    groups = -(-D // group)
    codes, scales, zero = np.zeros((N, D)), torch.zeros(N, groups, dtype=scales_dtype), np.full((N, groups), 8.0)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        for g in range(groups):
            v = w64[:, g * group:(g + 1) * group]
            f = np.where(np.isfinite(v), v, 0.0)
            if zeros:
                low, high = np.minimum(f.min(axis=1), 0.0), np.maximum(f.max(axis=1), 0.0)
                width = (high - low).astype(np.float32).astype(np.float64)
                width = np.where(np.isfinite(width), width, high - low)
                s = torch.from_numpy((width / 15.0).astype(np.float32)).to(scales_dtype)
            else:
                s = torch.from_numpy((np.abs(f).max(axis=1) / 7.0).astype(np.float32)).to(scales_dtype)
            scales[:, g] = s
            s = s.double().numpy()
            if zeros:
                zero[:, g] = np.where(s > 0, np.clip(np.round(-low / s), 0, 15), 8.0)
            q = np.clip(np.round(v / s[:, None]) + zero[:, g:g + 1], 0, 15)
            codes[:, g * group:(g + 1) * group] = np.where((s[:, None] > 0) & ~np.isnan(v), q, zero[:, g:g + 1])
    return codes, scales, zero


def check_quantize(out, w, group, zeros, scales_dtype):
    codes, scales, zero = quantize(w, group, zeros, scales_dtype)
    assert torch.equal(out["scales"].cpu(), scales)
    if zeros:
        np.testing.assert_array_equal(out["zeros"].cpu().numpy(), zero)
    D = w.shape[1]
    np.testing.assert_array_equal(codes_of(out["codes"], D), codes)
    if D % 2:
        assert (out["codes"].cpu().numpy()[:, -1] >> 4 == 0).all()


def check_matvec(out, x, codes, scales, zeros, group):
    """Every output against the formula.  A group's sum starts at (16 + zero) times the sum of its x and takes G products (16 + q) x;
    what is there on the way is at most the start and a few times the root of the products' squares.  Each of the G additions and of those
    of x's sum (16 at most) is off by a step of fp32 at most (a matrix instruction may cut where it adds), in either direction: six times the
    root of their squares, over all groups.  The sum of the groups: an addition a group; the output: half a step of its type."""
    D = x.shape[1]
    w = values(codes, scales, zeros, D, group)
    x64 = x.detach().cpu().double().numpy()
    want = x64 @ w.T
    q = codes_of(codes, D)
    s = scales.detach().cpu().double().numpy()
    groups = s.shape[1]
    square, ends = np.zeros(want.shape), np.zeros(want.shape)
    for g in range(groups):
        at = slice(g * group, min(D, (g + 1) * group))
        z = 8.0 if zeros is None else zeros.detach().cpu().double().numpy()[None, :, g]
        start = (16.0 + z) * np.abs(x64[:, at].sum(axis=1))[:, None]
        way = start + 4.0 * np.sqrt((x64[:, at] ** 2) @ ((16.0 + q[:, at]) ** 2).T)
        square += (group + 16) * (np.abs(s[None, :, g]) * way) ** 2
        ends += (x64[:, at] @ w[:, at].T) ** 2
    tol = 6.0 * 2.0 ** -23 * np.sqrt(square) + 6.0 * 2.0 ** -24 * np.sqrt(groups * ends) + 1.01 * STEP[out.dtype] * np.abs(want) + 2.0 ** -126
    got = out.detach().cpu().double().numpy()
    far = np.abs(got - want) - tol
    assert far.size == 0 or far.max() <= 0, (far.max(), got.flat[far.argmax()], want.flat[far.argmax()])
