"""Plain 64-bit forms of the operators of several continuations, on the CPU, and the error bounds that their arithmetic
allows."""
import numpy as np
import torch

from tests.operators_ref import F32, HALF

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def frequencies(hd, base=10000.0):
    return torch.tensor([base ** (-2.0 * j / hd) for j in range(hd // 2)], dtype=torch.float64)


def rotate(x, pos, freq, kind):
    """x [rows][heads][hd] turned to its positions, and the error that a result of type `kind` may have.

    Cosine and sine are off by what is left of the angle in fp32 (half a turn's half step: 2^-25 turns, 2^-22.3) and the
    function's own two steps of 2^-24 or less, together under 2^-21.8, and the two products' and the sum's
    roundings, under 2^-22.4 of each term; the angle itself by 2^-51 of the position (both sides form it in 64 bits).
    Then one rounding to `kind`."""
    half = x.shape[2] // 2
    a = pos.double()[:, None] * freq
    c, s = a.cos()[:, None], a.sin()[:, None]
    p, q = x.double()[..., :half], x.double()[..., half:]
    out = torch.cat([p * c - q * s, q * c + p * s], 2)
    size = (p.abs() + q.abs()).repeat(1, 1, 2)
    off = size * (2.0 ** -21 + pos.double().abs()[:, None, None] * 2.0 ** -51)
    step = (HALF * out.abs()).clamp_min(2.0 ** -25) if kind == "f16" else F32 * out.abs()
    return out, off * 1.01 + step


def candidates(x, scores, ended=None, end=None):
    """[beams][vocab] values in float64 of one group: logits x, scores [beams], ended [beams]."""
    x, scores = np.asarray(x, np.float64), np.asarray(scores, np.float64)
    out = np.full(x.shape, -np.inf)
    for b in range(len(x)):
        if not np.isfinite(scores[b]):
            continue
        if ended is not None and ended[b]:
            out[b, end] = scores[b]
            continue
        m = x[b].max()
        if not np.isfinite(m):               # NaN, +inf, or nothing but -inf
            continue
        out[b] = scores[b] + (x[b] - (m + np.log(np.exp(x[b] - m).sum())))
    return out


def select(values, n):
    """(values, beams, tokens) of the n first candidates of a group: larger values first, then the lower beam and token."""
    flat = values.reshape(-1)
    at = np.argsort(-flat, kind="stable")[:n]
    return flat[at], at // values.shape[1], at % values.shape[1]


def value_bound(v):
    """Largest error of a candidate's value: sums of at most 32 exponentials one after the other in fp32 (the rest in
    64 bits), each exponential off by its argument's roundings (of at most 16 where it counts) and two steps, all of
    one sign, so absolute behind the logarithm; and the value's own rounding to fp32."""
    return (32 + 16 + 12) * F32 + F32 * np.abs(np.where(np.isfinite(v), v, 0))


def check_group(score, parent, token, values, n):
    """A group's outputs against its candidates' values: order, ties and values.  Candidates whose values are nearer to
    each other than the bound may change places, others not; equal ones (in 64 bits, of equal logits) never."""
    want, wb, wt = select(values, n)
    got = values[parent, token]
    assert len({(int(b), int(t)) for b, t in zip(parent, token)}) == n, "a candidate twice"
    with np.errstate(invalid="ignore"):
        far = np.abs(got - want)
    far = np.where(np.isneginf(got) & np.isneginf(want), 0, far)
    bound = value_bound(want)
    assert (far <= 2 * bound).all(), (got, want)
    same = (parent == wb) & (token == wt)
    assert (same | (far > 0)).all(), "ties go to the lower beam, then to the lower token"
    err = np.abs(np.where(np.isneginf(got), 0, score.astype(np.float64) - np.where(np.isneginf(got), 0, got)))
    assert (np.isneginf(score) == np.isneginf(got)).all() and (err <= bound).all(), (score, got)
