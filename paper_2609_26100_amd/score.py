"""Scores of given continuations of a prefilled sequence: log probabilities of
their tokens under the verifier, as tasks with several given answers need them
(the answer is the most probable one).

The continuations go through the decoder together: the sequence is forked to
scratch sequences, one for each continuation of a group, and one batched verify
of chains (root, then the continuation without its last token) reads every
block's weights once for all of them; node i's logits give the log probability
of token i.  Nothing is committed to the sequence itself, and the forks take its
skip mask and attention window.
"""
from __future__ import annotations

import numpy as np


def _tokens(c, vocab):
    """A continuation as an int32 array; every token is checked here, for the last one never goes through the decoder."""
    t = np.asarray(c)
    if t.ndim != 1 or not len(t):
        raise ValueError("a continuation is a list of at least one token")
    if not ((t >= 0) & (t < vocab) & (t == np.floor(t))).all():
        raise ValueError("a continuation holds a token outside the vocabulary")
    return np.ascontiguousarray(t, dtype=np.int32)


def continuation_logprobs(verifier, seq, root, continuations, scratch):
    """Log probabilities of each continuation's tokens, one float32 array a continuation.

    root: the last prompt token, whose K/V are not cached yet.  scratch: sequences of the verifier, other than seq,
    whose contents may be replaced; up to min(len(scratch), max_batch) continuations share a step.  Continuations longer
    than a step's rows go through several steps.  A token outside the vocabulary is refused (ValueError)."""
    scratch = list(dict.fromkeys(int(s) for s in scratch))
    if not scratch or seq in scratch:
        raise ValueError("scoring needs scratch sequences other than the scored one")
    conts = [_tokens(c, verifier.cfg.vocab) for c in continuations]
    out = [np.empty(len(c), np.float32) for c in conts]
    cfg = verifier.cfg
    rows = min(cfg.max_nodes * cfg.max_batch, 128 if verifier.shape.dtype == "bf16" else 64)
    most = min(len(scratch), cfg.max_batch, rows)
    for g0 in range(0, len(conts), most):
        group = range(g0, min(g0 + most, len(conts)))
        ids = scratch[:len(group)]
        verifier.fork(seq, ids)
        roots, done = {i: int(root) for i in group}, {i: 0 for i in group}
        live = list(group)
        while live:
            room = min(cfg.max_nodes, rows // len(live))
            n = [min(room, len(conts[i]) - done[i]) for i in live]
            given = [conts[i][done[i]:done[i] + k] for i, k in zip(live, n)]
            chains = [np.concatenate([[roots[i]], t[:-1]]).astype(np.int32) for i, t in zip(live, given)]
            verifier.verify_batch([ids[i - g0] for i in live], chains)
            lp = verifier.logprobs(sum(n), np.concatenate(given))[0]
            at = 0
            for i, k, t, c in zip(live, n, given, chains):
                out[i][done[i]:done[i] + k] = lp[at:at + k]
                at += k
                done[i] += k
                if done[i] < len(conts[i]):        # the rest follows behind these tokens
                    verifier.prefill(ids[i - g0], c)
                    roots[i] = int(t[-1])
            live = [i for i in live if done[i] < len(conts[i])]
    return out


def choose(verifier, seq, root, choices, scratch, per_token=False):
    """(index of the most probable choice, score of each): the sum of its tokens' log probabilities, or with per_token
    their mean; the first of equal ones.  A score of NaN (from logits that are not finite) loses to every other."""
    lps = continuation_logprobs(verifier, seq, root, choices, scratch)
    scores = np.asarray([lp.mean(dtype=np.float64) if per_token else lp.sum(dtype=np.float64) for lp in lps])
    return int(np.argmax(np.where(np.isnan(scores), -np.inf, scores))), scores
