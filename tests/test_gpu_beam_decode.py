"""Beam search with the verifier: forks, batched steps, the choice of beams and the reordering of sequences, against a plain
64-bit forward."""
import numpy as np
import pytest
import torch

import synth
from paper_2609_26100_amd import ops
from paper_2609_26100_amd import tss as abi
from paper_2609_26100_amd.decode import autoregressive_decode, beam_decode
from tests import beams_ref, window_ref
from tests.gpu_common import TOL, gpu_verifier

pytestmark = pytest.mark.gpu

TINY = synth.TINY
SMALL = synth.ModelShape("small-3L-d512", 91, n_layers=3, d_model=512, n_heads=4, head_dim=128, ffn_dim=1408, vocab=4096)
SHAPES = {"f32": TINY, "bf16": SMALL}


@pytest.fixture(scope="module")
def models():
    made = {}

    def get(kind):
        if kind not in made:
            s = SHAPES[kind]
            v = gpu_verifier(s, random_gains=True, n_seqs=10, max_tokens=400, max_nodes=64, max_batch=8)
            made[kind] = (v, window_ref.Model(s))
        return made[kind]
    yield get
    for v, _ in made.values():
        v.close()


def start(v, seq, ctx, window=(0, 0), mask=None):
    v.truncate(seq, 0)
    v.set_mask(seq, mask)
    v.set_window(seq, *window)
    v.prefill(seq, ctx)


@pytest.mark.parametrize("kind,window,skip,n", [
    ("f32", (0, 0), [], 4), ("f32", (4, 64), [], 3), ("f32", (0, 0), [2], 8), ("bf16", (0, 0), [], 4),
    ("bf16", (4, 64), [1], 5), ("f32", (0, 0), [], 1)])
def test_every_step_against_64_bits(models, kind, window, skip, n):
    """The beams of k steps are the best continuations, by the 64-bit forward, of the beams of k - 1 steps; no other
    candidate is better by more than the logits' tolerance allows."""
    v, m = models(kind)
    s = SHAPES[kind]
    prompt = synth.context_tokens(s.vocab, 83, stream=300)
    start(v, 9, prompt[:-1], window, synth.mask_from_layers(s.n_layers, skip) if skip else None)
    tol = 2 * TOL[s.dtype][0]                        # of a log probability: the logit's and the sum's

    def lp(tokens):                                  # of every next token
        full = np.concatenate([prompt, tokens])
        x = m.logits(full, np.arange(len(full)), window_ref.context_see(len(full), *window), skip)[-1]
        return beams_ref.candidates(x[None], [0.0])[0]
    live = {(): 0.0}
    for k in range(1, 6):
        r = beam_decode(v, 9, int(prompt[-1]), k, list(range(n)))
        assert r.steps == k and len(r.tokens) == n and (np.diff(r.scores) <= 0).all()
        values = {}
        for t, score in live.items():
            x = lp(np.array(t, np.int32))
            for i in np.argsort(-x, kind="stable")[: 2 * n + 1]:
                values[t + (int(i),)] = score + x[i]
        best = sorted(values.values(), reverse=True)
        got = {}
        for t, score in zip(r.tokens, r.scores):
            t = tuple(int(i) for i in t)
            assert t[:-1] in live and t not in got
            got[t] = live[t[:-1]] + lp(np.array(t[:-1], np.int32))[t[-1]]
            assert abs(got[t] - score) <= k * tol
            assert got[t] >= best[n - 1] - 2 * k * tol
        live = got
    assert v.length(9) == 82


def test_one_beam_is_greedy_decoding(models):
    v, _ = models("f32")
    prompt = synth.context_tokens(TINY.vocab, 50, stream=301)
    start(v, 0, prompt[:-1])
    r = beam_decode(v, 0, int(prompt[-1]), 30, [3])
    want = autoregressive_decode(v, 0, int(prompt[-1]), 30, logprobs=0)
    np.testing.assert_array_equal(r.tokens[0], want.tokens)
    assert abs(r.scores[0] - want.logprobs.logprob.sum()) < 1e-3


def test_nothing_cached_before_the_root(models):
    v, _ = models("f32")
    for q in range(4):
        v.truncate(q, 0)
        v.set_window(q, 0, 0)
        v.set_mask(q, None)
    r = beam_decode(v, 0, 7, 20, [3])
    want = autoregressive_decode(v, 0, 7, 20)
    np.testing.assert_array_equal(r.tokens[0], want.tokens)
    v.truncate(0, 0)
    three = beam_decode(v, 0, 7, 20, [1, 2, 3])
    assert (np.diff(three.scores) <= 0).all() and len(three.tokens[0]) == 20 and v.length(0) == 0


def test_ended_beams(models):
    """A beam that ends keeps its score, and the search stops when all have ended."""
    v, _ = models("f32")
    prompt = synth.context_tokens(TINY.vocab, 40, stream=302)
    start(v, 0, prompt[:-1])
    free = beam_decode(v, 0, int(prompt[-1]), 4, [1, 2, 3])
    end = int(free.tokens[0][1])                     # ends the best beam behind two tokens
    r = beam_decode(v, 0, int(prompt[-1]), 4, [1, 2, 3], end_token=end)
    for t, score, over in zip(r.tokens, r.scores, r.ended):
        assert over == (t[-1] == end) and (t[:-1] != end).all() and (over or len(t) == 4)
    two = beam_decode(v, 0, int(prompt[-1]), 2, [1, 2, 3])
    i = next(i for i, t in enumerate(two.tokens) if t[-1] == end)
    j = next(j for j, t in enumerate(r.tokens) if len(t) == 2 and (t == two.tokens[i]).all())
    assert r.ended[j] and abs(r.scores[j] - two.scores[i]) < 1e-5
    greedy = autoregressive_decode(v, 0, int(prompt[-1]), 4).tokens
    start(v, 0, prompt[:-1])
    one = beam_decode(v, 0, int(prompt[-1]), 30, [1], end_token=int(greedy[2]))
    n = list(greedy).index(greedy[2]) + 1
    assert one.ended[0] and one.steps == n and list(one.tokens[0]) == list(greedy[:n])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_reorder_sequences(models, kind):
    """Lengths, masks, windows and tokens move with their sequence, exchanges and all."""
    v, _ = models(kind)
    s = SHAPES[kind]
    prompt = synth.context_tokens(s.vocab, 37, stream=303)
    start(v, 0, prompt)
    v.fork(0, [1, 2, 3, 4])
    masks = [None, [1], None, [0, 2], None]
    for q in range(5):
        v.set_mask(q, synth.mask_from_layers(s.n_layers, masks[q]) if masks[q] else None)
        v.set_window(q, q, 64 * (q % 2))
        v.prefill(q, synth.context_tokens(s.vocab, 5 + 20 * q, stream=310 + q))
    probe = synth.context_tokens(s.vocab, 3, stream=320)

    def state(q):
        v.verify(q, probe)
        return v.length(q), v.logits(3)
    before = [state(q) for q in range(5)]
    assert len({b[0] for b in before}) == 5
    for parents in ([1, 0, 2, 4, 3], [2, 2, 0, 0, 4], [4, 3, 2, 1, 0]):
        v.reorder([0, 1, 2, 3, 4], parents, 37)
        v.check_kv()
        before = [before[p] for p in parents]
        for q in range(5):
            n, x = state(q)
            assert n == before[q][0]
            np.testing.assert_array_equal(x, before[q][1])
    v.reorder([3], [0])                              # one sequence alone
    assert state(3)[0] == before[3][0]
    v.truncate(2, 0)
    v.reorder([2, 4], [1, 0])                        # nothing in one of them
    assert v.length(4) == 0 and state(2)[0] == before[4][0]
    np.testing.assert_array_equal(state(2)[1], before[4][1])


def test_beams_of_a_step(models):
    """The same as the operator on the step's logits, and they stay as they are."""
    v, _ = models("f32")
    for q in range(6):
        start(v, q, synth.context_tokens(TINY.vocab, 20 + q, stream=330 + q))
    al, nt = v.verify_batch(list(range(6)), [[q] for q in range(6)])
    lg = v.logits_device(6)
    scores = -np.arange(6, dtype=np.float32).reshape(2, 3)
    ended = np.array([[0, 1, 0], [0, 0, 0]])
    for e in (None, ended):
        got = v.beams(scores, 6, e, 7)
        want = ops.beam_select(lg, torch.from_numpy(scores).cuda(), 6,
                               None if e is None else torch.from_numpy(e.astype(np.int32)).cuda(), 7)
        for a, b in zip(got, want):
            np.testing.assert_array_equal(a, b.cpu().numpy())
    assert torch.equal(v.logits_device(6), lg)
    a2, n2 = v.verify_batch(list(range(6)), [[q] for q in range(6)])    # the scratch is the step's own again
    np.testing.assert_array_equal(n2, nt)
    assert torch.equal(v.logits_device(6), lg)


def test_refusals(models):
    v, _ = models("f32")
    start(v, 0, synth.context_tokens(TINY.vocab, 20, stream=340))
    v.fork(0, [1, 2])
    for bad in (([0, 1], [0, 2], 0), ([0, 1], [-1, 0], 0), ([0, 0], [0, 1], 0), ([0, 10], [0, 1], 0), ([], [], 0),
                ([0, 1], [1, 0], 21), ([0, 1], [1, 0], -1)):
        with pytest.raises(abi.TSSError) as e:
            v.reorder(*bad)
        assert e.value.status == abi.TSS_EINVAL
    with pytest.raises(ValueError):
        v.reorder([0, 1], [0])
    v.verify_batch([0, 1], [[1], [2]])
    s = np.zeros((1, 2), np.float32)
    for bad in ((np.zeros((1, 3), np.float32), 2), (np.zeros((2, 2), np.float32), 2), (s, 0), (s, 65),
                (s, 2, np.zeros((1, 2), np.int32), TINY.vocab), (s, 2, np.zeros((1, 2), np.int32), -1)):
        with pytest.raises(abi.TSSError) as e:
            v.beams(*bad)
        assert e.value.status == abi.TSS_EINVAL
    for bad in ((np.zeros(2, np.float32), 2), (s, 2, np.zeros(2, np.int32)), (s, 2.5)):
        with pytest.raises(ValueError):
            v.beams(*bad)
    for bad in (dict(beams=[]), dict(beams=[0, 1]), dict(beams=[1, 1]), dict(beams=list(range(1, 10))),
                dict(end_token=TINY.vocab), dict(end_token=-1), dict(max_new=381), dict(beams=[1.5])):
        with pytest.raises(ValueError):
            beam_decode(v, 0, 1, **dict(dict(max_new=3, beams=[1, 2]), **bad))
    assert v.length(0) == 20
    r = beam_decode(v, 0, 1, 0, [1, 2])
    assert r.steps == 0 and [len(t) for t in r.tokens] == [0, 0]
