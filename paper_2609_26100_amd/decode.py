"""Decode loops around the sparse verifier.

speculative_decode: greedy speculative decoding of one sequence (Problem
Formulation): a drafter proposes a chain or tree after the last committed
token, one verify step under the request's skip mask accepts the longest root
path that matches the verifier's greedy tokens and commits it with the bonus
token, and the bonus token becomes the next root.  With greedy acceptance
the output is exactly what plain greedy decoding with the same verifier
produces, however good the drafts are; only the number of verify steps
changes.

autoregressive_decode: the plain greedy loop, one token per verify step (a
one-node draft: the root alone), the baseline both for the output and for
throughput.

beam_decode: beam search under the request's skip mask and window.  The beams are
forks of the sequence that go through the decoder together, one node each in a
batched step; the best continuations are chosen from the step's logits on the device
and the beams' cached tokens behind the prompt are reordered in place.

A drafter is any callable drafter(root, pos) -> (tokens, parent) with
tokens[0] == root, parent[0] == -1 (parent None = chain), where pos counts
the tokens generated so far.  The loop's own host work per step is a
verify call, reading the accepted path, and list appends; with `logprobs` also
one call that computes the emitted tokens' log probabilities from the step's
logits.
"""
from __future__ import annotations

import time
from dataclasses import dataclass, field

import numpy as np

from . import tss as abi


@dataclass
class DecodeLogprobs:
    logprob: np.ndarray            # of each generated token
    entropy: np.ndarray            # of the distribution that it was taken from, nats
    top_logprob: np.ndarray        # [tokens][k] alternatives, most likely first
    top_token: np.ndarray


class _Logprobs:
    """Collects the log probabilities of the emitted tokens, step by step."""

    def __init__(self, verifier, k):
        if k not in range(min(abi.TSS_LOGPROBS_MAX_TOP, verifier.cfg.vocab) + 1):  # before the first step commits
            raise ValueError("logprobs must be None or from 0 to min(32, vocab) alternatives")
        self.verifier, self.k, self.parts = verifier, int(k), []

    def add(self, n_nodes, nodes, emitted):
        """`emitted` follow `nodes` of the last verify, which had n_nodes."""
        given = np.full(n_nodes, -1, dtype=np.int32)
        given[nodes] = emitted
        lp, _, ent, tl, tt = self.verifier.logprobs(n_nodes, given, self.k)
        none = np.empty((len(nodes), 0))
        self.parts.append((lp[nodes], ent[nodes], tl[nodes] if self.k else none, tt[nodes] if self.k else none))

    def result(self, n):
        if not self.parts:
            return DecodeLogprobs(np.empty(0, np.float32), np.empty(0, np.float32), np.empty((0, self.k), np.float32),
                                  np.empty((0, self.k), np.int32))
        a, b, c, d = (np.concatenate(x)[:n] for x in zip(*self.parts))
        return DecodeLogprobs(a, b, c.astype(np.float32), d.astype(np.int32))


@dataclass
class DecodeResult:
    tokens: np.ndarray             # the first max_new generated tokens
    steps: int                     # verify steps
    accept_lens: list = field(default_factory=list)  # accepted draft tokens per step
    seconds: float = 0.0           # wall time of the loop
    draft_seconds: float = 0.0     # of which in the drafter
    logprobs: DecodeLogprobs | None = None  # of the tokens, where asked for

    @property
    def tokens_per_step(self):
        return (sum(self.accept_lens) + len(self.accept_lens)) / max(1, self.steps)

    @property
    def tokens_per_second(self):
        return len(self.tokens) / self.seconds if self.seconds > 0 else float("nan")


def speculative_decode(verifier, seq, root, max_new, drafter, mask=None, logprobs=None):
    """Generates at least max_new tokens after `root` (the last prompt token,
    whose K/V are not cached yet) and returns the first max_new.  Every step
    commits, so the sequence grows by accept_len + 1 per step (up to one
    step's worth beyond max_new).  logprobs: None, or how many alternatives
    (0 to 32) the result's log probabilities come with."""
    out, acc = [], []
    lps = None if logprobs is None else _Logprobs(verifier, logprobs)
    t_draft = 0.0
    t0 = time.perf_counter()
    while len(out) < max_new:
        a = time.perf_counter()
        tokens, parent = drafter(root, len(out))
        t_draft += time.perf_counter() - a
        al, nt = verifier.verify(seq, tokens, parent, mask=mask, commit=True)
        if al:
            if parent is None:
                out.extend(int(t) for t in tokens[1:al + 1])
            else:
                out.extend(int(tokens[j]) for j in verifier.path(0)[1:])
        out.append(int(nt))
        if lps is not None:
            nodes = list(range(al + 1)) if parent is None else [int(j) for j in verifier.path(0)]
            lps.add(len(tokens), nodes, out[-al - 1:])
        acc.append(int(al))
        root = int(nt)
    return DecodeResult(np.asarray(out[:max_new], dtype=np.int32), len(acc), acc, time.perf_counter() - t0, t_draft,
                        lps.result(max_new) if lps is not None else None)


def autoregressive_decode(verifier, seq, root, max_new, mask=None, logprobs=None):
    """Plain greedy decoding: one committing verify of the root alone per token (logprobs as speculative_decode)."""
    out = []
    lps = None if logprobs is None else _Logprobs(verifier, logprobs)
    one = np.zeros(1, dtype=np.int32)
    t0 = time.perf_counter()
    for _ in range(max_new):
        one[0] = root
        _, nt = verifier.verify(seq, one, None, mask=mask, commit=True)
        out.append(int(nt))
        if lps is not None:
            lps.add(1, [0], [int(nt)])
        root = int(nt)
    return DecodeResult(np.asarray(out, dtype=np.int32), max_new, [0] * max_new, time.perf_counter() - t0,
                        logprobs=lps.result(max_new) if lps is not None else None)


@dataclass
class BeamResult:
    tokens: list                   # of each beam, the best first: int32 arrays, up to and with end_token
    scores: np.ndarray             # sums of the tokens' log probabilities
    ended: np.ndarray              # whether the beam ends with end_token
    steps: int


def beam_decode(verifier, seq, root, max_new, beams, end_token=None):
    """Beam search after `root` (the last prompt token, whose K/V are not cached yet): the len(beams) most probable
    continuations found, of at most max_new tokens, or shorter ones that end with end_token.

    beams: sequences of the verifier, other than seq, whose contents may be replaced, one for each beam, at most
    max_batch.  They take seq's skip mask and window; seq itself stays as it is.  A score of -inf is no continuation
    (fewer tokens with a finite logit than beams).  What the beams' sequences hold afterwards is not the returned tokens
    (the last step is neither committed nor reordered): to go on, fork seq again and prefill those."""
    beams = [int(s) for s in abi._int32s(beams, "beams")]
    n = len(beams)
    if not 1 <= n <= min(verifier.cfg.max_batch, abi.TSS_BEAMS_MAX) or len(set(beams)) < n or seq in beams:
        raise ValueError("beams must be from 1 to max_batch different sequences other than the decoded one")
    vocab = verifier.cfg.vocab
    if end_token is not None and not 0 <= end_token < vocab:
        raise ValueError("end_token outside the vocabulary")
    base = verifier.length(seq)
    if base + max_new > verifier.max_tokens:
        raise ValueError("the beams' sequences have no room for that many tokens")
    verifier.fork(seq, beams)
    scores = np.full((1, n), -np.inf, np.float32)
    scores[0, 0] = 0
    ended = np.zeros((1, n), np.int32)
    history = np.empty((n, 0), np.int32)
    roots = np.full(n, root, np.int32)
    steps = 0
    while steps < max_new and not ended.all():
        verifier.verify_batch(beams, list(roots[:, None]), commit=steps + 1 < max_new)
        scores, parent, roots = verifier.beams(scores, n, None if end_token is None else ended, end_token or 0)
        parent, roots = parent[0], roots[0]
        steps += 1
        if steps < max_new:
            verifier.reorder(beams, parent, base)
        history = np.concatenate([history[parent], roots[:, None]], 1)
        if end_token is not None:
            ended = (ended[:, parent] != 0) | (roots == end_token)[None]
            ended = ended.astype(np.int32)
    tokens = []
    for h in history:
        at = np.flatnonzero(h == end_token) if end_token is not None else ()
        tokens.append(h[: at[0] + 1].copy() if len(at) else h.copy())
    return BeamResult(tokens, scores[0], ended[0] != 0, steps)
