"""Plain 64-bit forms of the operators, on the CPU, and the error bounds that their arithmetic allows."""
import numpy as np
import torch

HALF = 2.0 ** -11        # half a step of fp16, relative
F32 = 2.0 ** -24         # half a step of fp32, relative


# --- log probabilities --------------------------------------------------------

def order(x):
    """Tokens of a row, first to last: larger logits first, the lower index among equal ones, NaN the largest."""
    key = np.where(np.isnan(x), np.inf, x)
    nan_first = ~np.isnan(x)
    return np.lexsort((np.arange(len(x)), -key, nan_first))


def logprobs(x):
    """(log probabilities, entropy) of one row in float64."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or np.isposinf(x).any():
        return np.full(len(x), np.nan), np.nan
    m = x.max()
    if np.isneginf(m):
        return np.full(len(x), -np.inf), 0.0
    e = np.exp(x - m)
    lp = x - m - np.log(e.sum())
    p = e / e.sum()
    return lp, float(-(p[p > 0] * lp[p > 0]).sum())


def logprob_bound(vocab, lp):
    """Largest error of a log probability: the sum's at most V / 256 + 32 additions one after the other (relative to a
    sum of positive terms, so absolute behind the logarithm) with each term's exponential (two steps and the rounding
    of its argument, which is at most 16 where the term counts), and the roundings of the subtractions."""
    return (vocab / 256 + 32 + 20) * F32 + 4 * F32 * (1 + np.abs(np.where(np.isfinite(lp), lp, 0)))


def entropy_bound(vocab, lp):
    """ln S - T / S: the bound of ln S, and T's terms (x - m) e^(x - m), of one sign, each within the same share."""
    p = np.exp(lp[np.isfinite(lp)])
    t = float((p * (lp[np.isfinite(lp)].max() - lp[np.isfinite(lp)])).sum()) if len(p) else 0.0
    return (vocab / 256 + 32 + 20) * F32 * (1 + 2 * t) + 8 * F32 * (1 + t + np.log(vocab))


# --- attention with a window and sinks ------------------------------------------

def visible(rows, length, sinks, window):
    """[rows][length]: what each of the last `rows` tokens sees (a row before token 0 sees nothing)."""
    p = torch.arange(length - rows, length)[:, None]
    t = torch.arange(length)[None]
    see = t <= p
    if window:
        see = see & ((t < sinks) | (t > p - window))
    return see


def attention(q, k, v, see, scale=None):
    """q [rows][heads][hd], k, v [tokens][kv heads][hd], see [rows][tokens]: (output, bound of the error) in float64
    for operands in q's type."""
    rows, heads, hd = q.shape
    group = heads // k.shape[1]
    scale = hd ** -0.5 if scale is None else scale
    half = q.dtype == torch.float16
    q, k, v = q.double(), k.double(), v.double()
    out = torch.zeros(rows, heads, hd, dtype=torch.float64)
    bound = torch.zeros_like(out)
    n = k.shape[0]
    some = see.any(1)
    for h in range(heads):
        kh, vh = k[:, h // group], v[:, h // group]
        s = (q[:, h] @ kh.T * scale).masked_fill(~see, -torch.inf)
        p = torch.nan_to_num(torch.softmax(s, 1), nan=0.0)
        o = p @ vh
        # a score's error: hd products summed in fp32, and the roundings of scaling and exponent
        d = ((q[:, h].abs() @ kh.T.abs() * scale) * see).amax(1) * (hd + 2) * F32
        d = d + (torch.where(see, s.abs(), 0.0).amax(1) + 8) * 4 * F32
        pv = p @ vh.abs()
        big = (see[:, :, None] * vh.abs()[None]).amax(1)
        # numerator and denominator both carry the scores' errors and those of n additions
        b = 2 * d[:, None] * pv * 1.1 + 2 * n * F32 * pv
        if half:  # probabilities in fp16 (those below its normal range to 2^-25), and the result's rounding
            b = b + HALF * pv + n * 2.0 ** -25 * big + HALF * o.abs() + 2.0 ** -25
        else:
            b = b + 2 * F32 * o.abs()
        out[:, h], bound[:, h] = o, b
    out[~some], bound[~some] = 0, 0
    return out, bound
