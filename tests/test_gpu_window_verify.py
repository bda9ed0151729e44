"""Verification steps, prompts, batches and sweeps of sequences with an attention window against a plain 64-bit forward, and
the operators together: windowed prompts, forks, batched steps and log probabilities."""
import dataclasses

import numpy as np
import pytest

import synth
from paper_2609_26100_amd import score
from paper_2609_26100_amd import tss as abi
from paper_2609_26100_amd.decode import autoregressive_decode, speculative_decode
from tests import operators_ref as ref
from tests import window_ref
from tests.gpu_common import TOL, gpu_verifier, log

pytestmark = pytest.mark.gpu

TINY = synth.TINY
# a bf16 decoder that takes prompts in passes, narrow enough for the 64-bit forward
SMALL = synth.ModelShape("small-3L-d512", 91, n_layers=3, d_model=512, n_heads=4, head_dim=128, ffn_dim=1408, vocab=4096)
SMALL64 = dataclasses.replace(SMALL, name="small-3L-hd64", shape_id=92, n_heads=8, head_dim=64)
SHAPES = {"f32": TINY, "bf16": SMALL, "bf16_64": SMALL64}


@pytest.fixture(scope="module")
def models():
    made = {}

    def get(kind):
        if kind not in made:
            s = SHAPES[kind]
            v = gpu_verifier(s, random_gains=True, n_seqs=10, max_tokens=2900, max_nodes=64, max_batch=8)
            made[kind] = (v, window_ref.Model(s))
        return made[kind]
    yield get
    for v, _ in made.values():
        v.close()


def start(v, seq, ctx, sinks, window, mask=None):
    v.truncate(seq, 0)
    v.set_mask(seq, mask)
    v.set_window(seq, sinks, window)
    v.prefill(seq, ctx)


def same(kind, got, want):
    err = float(np.max(np.abs(got - want)))
    assert err <= TOL[SHAPES[kind].dtype][0], err
    return err


@pytest.mark.parametrize("kind,n_ctx,nodes,tree,sinks,window,skip", [
    ("f32", 40, 6, False, 0, 64, []),          # nothing hidden yet
    ("f32", 200, 1, False, 4, 64, []),
    ("f32", 300, 17, True, 1, 100, [1]),
    ("f32", 301, 61, True, 33, 64, []),
    ("f32", 63, 64, False, 0, 64, []),
    ("bf16", 200, 1, False, 4, 64, []),
    ("bf16", 500, 6, False, 4, 129, []),
    ("bf16", 700, 16, True, 0, 200, [0]),
    ("bf16", 701, 17, True, 17, 64, []),
    ("bf16", 1500, 64, True, 4, 1000, []),
    ("bf16", 2600, 33, True, 4, 512, []),      # two passes of the prompt
    ("bf16", 65, 5, False, 0, 64, []),
    ("bf16_64", 400, 9, True, 3, 80, []),
    ("bf16_64", 901, 40, True, 16, 256, [2]),
])
def test_step_under_a_window(models, kind, n_ctx, nodes, tree, sinks, window, skip):
    v, m = models(kind)
    s = SHAPES[kind]
    ctx = synth.context_tokens(s.vocab, n_ctx, stream=n_ctx)
    draft = synth.context_tokens(s.vocab, nodes, stream=nodes + 1)
    parent = synth.random_tree(nodes, stream=nodes, max_children=3) if tree else None
    start(v, 0, ctx, sinks, window, synth.mask_from_layers(s.n_layers, skip))
    want = window_ref.step_logits(m, ctx, draft, parent, sinks, window, set(skip))
    for _ in range(2):                          # captured, then replayed
        al, nt = v.verify(0, draft, parent)
        e = same(kind, v.logits(nodes), want)
    log(f"{kind} {n_ctx} tokens, {nodes} nodes, sinks {sinks}, window {window}: {e:.2e}, split {v.attn_split()}")
    assert [r for _, r in v.attn_split()] == [nodes]
    st = abi.tss_verify_static(v.ctx, 0, draft, parent)
    assert st == (al, nt)
    same(kind, v.logits(nodes), want)
    v.check_kv()


def test_window_that_hides_nothing_and_back(models):
    v, m = models("bf16")
    ctx = synth.context_tokens(SMALL.vocab, 300, stream=1)
    draft = synth.context_tokens(SMALL.vocab, 5, stream=2)
    start(v, 0, ctx, 0, 0)
    v.verify(0, draft)
    plain = v.logits(5)
    v.set_window(0, 0, 2900)                    # the capacity: the same as none, bit by bit
    v.verify(0, draft)
    np.testing.assert_array_equal(v.logits(5), plain)
    v.set_window(0, 7, 400)                     # longer than the context
    v.verify(0, draft)
    same("bf16", v.logits(5), plain)
    v.set_window(0, 4, 64)
    v.verify(0, draft)
    assert np.abs(v.logits(5) - plain).max() > 1e-3
    v.set_window(0, 0, 0)
    v.verify(0, draft)
    np.testing.assert_array_equal(v.logits(5), plain)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_one_shape_as_the_context_grows(models, kind):
    """A captured step follows a context that grows past its window; committed steps equal the 64-bit forward."""
    v, m = models(kind)
    s = SHAPES[kind]
    ctx = synth.context_tokens(s.vocab, 100, stream=7)
    start(v, 0, ctx, 4, 64)
    seen = list(ctx)
    for step in range(4):
        draft = synth.context_tokens(s.vocab, 3, stream=30 + step)
        want = window_ref.step_logits(m, np.array(seen), draft, None, 4, 64)
        al, _ = v.verify(0, draft, commit=True)
        same(kind, v.logits(3), want)
        seen += list(draft[: al + 1])
        more = synth.context_tokens(s.vocab, 41, stream=60 + step)   # a chunk of up to 64
        v.prefill(0, more)
        seen += list(more)
        assert v.length(0) == len(seen)


@pytest.mark.parametrize("kind,n_seqs,nodes", [("f32", 3, 9), ("bf16", 4, 5), ("bf16", 8, 16), ("bf16", 2, 64)])
def test_batch_of_windows(models, kind, n_seqs, nodes):
    """Sequences with windows of their own, one of them with none, one with another mask."""
    v, m = models(kind)
    s = SHAPES[kind]
    windows = [(4, 64), (0, 0), (20, 100), (0, 300)]
    seqs, ctxs, drafts, wants = list(range(n_seqs)), [], [], []
    for i in seqs:
        sinks, window = windows[i % 4]
        skip = [1] if i == 2 else []
        ctxs.append(synth.context_tokens(s.vocab, 90 + 150 * (i % 3) + i, stream=100 + i))
        start(v, i, ctxs[i], sinks, window, synth.mask_from_layers(s.n_layers, skip))
        drafts.append(synth.context_tokens(s.vocab, nodes, stream=120 + i))
        wants.append(window_ref.step_logits(m, ctxs[i], drafts[i], None, sinks, window, set(skip)))
    for _ in range(2):
        v.verify_batch(seqs, drafts)
        got = v.logits(n_seqs * nodes)
        for i in seqs:
            same(kind, got[i * nodes:(i + 1) * nodes], wants[i])


def test_sweep_under_a_window(models):
    v, m = models("bf16")
    ctx = synth.context_tokens(SMALL.vocab, 260, stream=140)
    start(v, 0, ctx, 4, 100)
    draft = synth.context_tokens(SMALL.vocab, 13, stream=141)
    masks = np.array([[(b >> l) & 1 for l in range(3)] for b in range(8)], np.uint8)
    acc, nxt = v.verify_sweep(0, draft, masks)
    for k in range(8):
        assert v.verify(0, draft, mask=masks[k])[0] == acc[k]
        same("bf16", v.logits(13), window_ref.step_logits(m, ctx, draft, None, 4, 100, set(np.flatnonzero(masks[k])),
                                                          dense_context=True))


def test_timing_of_windowed_attention(models):
    """One attention launch a step is timed, its merge launch is not taken for another."""
    v, _ = models("bf16")
    start(v, 0, synth.context_tokens(SMALL.vocab, 1500, stream=145), 4, 1000)
    draft = synth.context_tokens(SMALL.vocab, 40, stream=146)
    v.verify(0, draft)
    want = v.logits(40)
    abi.tss_profile_kernel(v.ctx, abi.TSS_K_ATTN, 1)
    abi.tss_profile_read(v.ctx, reset=True)
    for _ in range(3):
        v.verify(0, draft)
    ms, n = abi.tss_profile_read(v.ctx, reset=True)
    abi.tss_profile_kernel(v.ctx, -1)
    assert n == 3 and 0 < ms < 3
    assert v.attn_split()[0][0] > 1              # merged across workgroups
    np.testing.assert_array_equal(v.logits(40), want)


def test_window_refusals(models):
    v, _ = models("f32")
    for bad in ((0, -1, 64), (0, 0, -1), (0, 0, 63), (0, 4, 1), (99, 0, 64), (-1, 0, 64)):
        with pytest.raises(abi.TSSError) as e:
            v.set_window(*bad)
        assert e.value.status == abi.TSS_EINVAL


# --- forks -----------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [None, 0, 1, 16, 37, 160])
def test_fork_is_the_source(models, kind, n):
    """A fork gives the source's logits bit by bit, under its mask and window, and leaves the source alone."""
    v, _ = models(kind)
    s = SHAPES[kind]
    ctx = synth.context_tokens(s.vocab, 333, stream=150)
    mask = synth.mask_from_layers(s.n_layers, [1])
    for sq in range(10):
        start(v, sq, synth.context_tokens(s.vocab, 20 + sq, stream=151), 0, 0)
    start(v, 3, ctx, 4, 100, mask)
    dsts = [7, 0, 9]
    v.fork(3, dsts, n)
    keep = 333 if n is None else n
    draft = synth.context_tokens(s.vocab, 6, stream=152)
    v.verify(3, draft)
    whole = v.logits(6)
    other = v.length(1)
    got = []
    for d in dsts:
        assert v.length(d) == keep
        v.verify(d, draft)
        got.append(v.logits(6))
    v.truncate(3, keep)
    v.verify(3, draft)
    want = v.logits(6)
    for g in got:
        np.testing.assert_array_equal(g, want)
    if keep == 333:
        np.testing.assert_array_equal(want, whole)
    # a fork goes its own way
    v.verify(7, draft, commit=True)
    v.prefill(7, synth.context_tokens(s.vocab, 30, stream=153))
    v.verify(3, draft)
    np.testing.assert_array_equal(v.logits(6), want)
    v.verify(9, draft)
    np.testing.assert_array_equal(v.logits(6), want)
    assert v.length(1) == other
    v.check_kv()


def test_fork_copies_what_the_source_holds(models):
    """Layers that the source skipped hold nothing in the fork either: a wider mask there is refused."""
    v, _ = models("f32")
    ctx = synth.context_tokens(TINY.vocab, 50, stream=160)
    start(v, 0, ctx, 0, 0, synth.mask_from_layers(TINY.n_layers, [2]))
    start(v, 1, ctx, 0, 0)
    v.fork(0, 1)
    with pytest.raises(abi.TSSError) as e:
        v.verify(1, [1, 2], mask=np.zeros(TINY.n_layers, np.uint8))
    assert e.value.status == abi.TSS_ESTATE
    v.verify(1, [1, 2])


def test_fork_long_context_to_many(models):
    """More page copies than one launch carries."""
    v, _ = models("bf16")
    ctx = synth.context_tokens(SMALL.vocab, 2800, stream=161)
    start(v, 0, ctx, 4, 64)
    v.fork(0, list(range(1, 10)))
    draft = synth.context_tokens(SMALL.vocab, 4, stream=162)
    v.set_window(0, 0, 0)
    v.verify(0, draft)
    want = v.logits(4)
    for d in range(1, 10):
        v.set_window(d, 0, 0)                   # every page of the fork is read
        v.verify(d, draft)
        np.testing.assert_array_equal(v.logits(4), want)


def test_fork_refusals(models):
    v, _ = models("f32")
    start(v, 0, synth.context_tokens(TINY.vocab, 20, stream=163), 0, 0)
    for src, dst, n in ((0, [0], 5), (0, [1, 1], 5), (0, [10], 5), (0, [-1], 5), (0, [1], 21), (0, [1], -1), (99, [1], 0),
                        (0, [], 5)):
        with pytest.raises(abi.TSSError) as e:
            v.fork(src, dst, n)
        assert e.value.status == abi.TSS_EINVAL
    assert v.length(0) == 20


# --- log probabilities of a step ----------------------------------------------------

def check_logprobs(lg, tokens, top, got):
    lp, rank, ent, tl, tt = got
    for r in range(len(lg)):
        want, e = ref.logprobs(lg[r])
        tol = ref.logprob_bound(lg.shape[1], want)
        o = ref.order(lg[r])
        assert abs(ent[r] - e) <= ref.entropy_bound(lg.shape[1], want)
        if tokens is not None:
            for j, t in enumerate(np.atleast_1d(tokens[r])):
                a, k = np.atleast_1d(lp[r])[j], np.atleast_1d(rank[r])[j]
                if 0 <= t < lg.shape[1]:
                    assert abs(a - want[t]) <= tol[t] and k == int(np.flatnonzero(o == t)[0])
                else:
                    assert np.isnan(a) and k == -1
        if top:
            np.testing.assert_array_equal(tt[r], o[:top])
            assert (np.abs(tl[r] - want[o[:top]]) <= tol[o[:top]]).all()


@pytest.mark.parametrize("kind,nodes,n,top", [("f32", 1, 1, 5), ("f32", 40, 0, 32), ("bf16", 6, 8, 0), ("bf16", 61, 1, 20)])
def test_logprobs_of_a_step(models, kind, nodes, n, top):
    v, _ = models(kind)
    s = SHAPES[kind]
    start(v, 0, synth.context_tokens(s.vocab, 70, stream=170), 0, 0)
    draft = synth.context_tokens(s.vocab, nodes, stream=171)
    rng = np.random.default_rng(nodes)
    tok = rng.integers(-1, s.vocab + 1, (nodes, n)).astype(np.int32) if n else None
    for again in range(2):
        al, nt = v.verify(0, draft)
        lg = v.logits(nodes)
        check_logprobs(lg, tok, top, v.logprobs(nodes, tok, top))
        np.testing.assert_array_equal(v.logits(nodes), lg)
        np.testing.assert_array_equal(v.greedy(nodes), lg.argmax(1))
    check_logprobs(lg[:1], None, 1, v.logprobs(1, None, 1))
    abi.tss_verify_static(v.ctx, 0, draft)
    check_logprobs(lg, tok, top, v.logprobs(nodes, tok, top))
    assert v.verify(0, draft) == (al, nt)       # the scratch they used is the step's own again
    np.testing.assert_array_equal(v.logits(nodes), lg)


def test_logprobs_after_a_static_step_leave_its_scratch_alone(models):
    """The library's static array is other contexts' too: what the call writes is in the context's own workspace."""
    v, _ = models("bf16")
    start(v, 0, synth.context_tokens(SMALL.vocab, 70, stream=173), 0, 0)
    draft = synth.context_tokens(SMALL.vocab, 9, stream=174)
    abi.tss_verify_static(v.ctx, 0, draft)
    v.torch.cuda.synchronize()
    before = v.workspace.clone()
    got = v.logprobs(9, draft, 4)
    changed = (v.workspace != before).sum().item()
    # given tokens, log probabilities, ranks, entropies, alternatives: words that differ from what was there
    assert changed > 9 * 8
    check_logprobs(v.logits(9), draft, 4, got)


def test_logprobs_refusals(models):
    v, _ = models("f32")
    start(v, 0, synth.context_tokens(TINY.vocab, 20, stream=172), 0, 0)
    v.verify(0, [1, 2, 3])
    for bad in ((0, None, 1), (4, None, 1), (3, None, 33), (3, None, -1), (3, np.zeros((3, 9), np.int32), 0)):
        with pytest.raises(abi.TSSError) as e:
            v.logprobs(*bad)
        assert e.value.status == abi.TSS_EINVAL
    with pytest.raises(ValueError):
        v.logprobs(3, np.zeros(2, np.int32))


def test_decoded_tokens_with_their_logprobs(models):
    """The tokens are those of a decode without; log probabilities agree between the loops and with the alternatives."""
    v, _ = models("f32")
    prompt = synth.context_tokens(TINY.vocab, 60, stream=180)

    def decode(fn, *args, **kw):
        start(v, 0, prompt[:-1], 4, 64)
        return fn(v, 0, int(prompt[-1]), 40, *args, **kw)
    plain = decode(autoregressive_decode)
    a = decode(autoregressive_decode, logprobs=3)
    np.testing.assert_array_equal(plain.tokens, a.tokens)
    assert plain.logprobs is None and a.logprobs.top_token.shape == (40, 3)
    np.testing.assert_array_equal(a.logprobs.top_token[:, 0], a.tokens)   # greedy: the first alternative
    np.testing.assert_array_equal(a.logprobs.top_logprob[:, 0], a.logprobs.logprob)

    def chain(root, pos):                        # right, right, wrong
        t = [root] + [int(plain.tokens[min(pos + i, 39)]) for i in range(2)]
        return np.array(t + [(t[-1] + 1) % TINY.vocab], np.int32), None

    def tree(root, pos):                         # a wrong child before the right one
        good = int(plain.tokens[min(pos, 39)])
        return np.array([root, (good + 1) % TINY.vocab, good], np.int32), np.array([-1, 0, 0], np.int32)
    for drafter in (chain, tree):
        b = decode(speculative_decode, drafter, logprobs=3)
        np.testing.assert_array_equal(b.tokens, plain.tokens)
        assert b.steps < 40
        assert np.abs(b.logprobs.logprob - a.logprobs.logprob).max() < 1e-4
        assert np.abs(b.logprobs.entropy - a.logprobs.entropy).max() < 1e-3
    c = decode(speculative_decode, chain, logprobs=0)
    assert c.logprobs.top_token.shape == (40, 0) and np.isfinite(c.logprobs.logprob).all()


# --- together ------------------------------------------------------------------------

@pytest.mark.parametrize("kind,window", [("f32", (4, 64)), ("bf16", (4, 100)), ("bf16", (0, 0))])
def test_scores_of_continuations(models, kind, window):
    """A windowed prompt, forked for its continuations, scored in batched steps: the 64-bit log probabilities."""
    v, m = models(kind)
    s = SHAPES[kind]
    prompt = synth.context_tokens(s.vocab, 210, stream=190)
    start(v, 2, prompt[:-1], *window)
    lens = [1, 5, 2, 33, 90, 7, 1, 20, 3, 64, 65]
    conts = [synth.context_tokens(s.vocab, n, stream=200 + i) for i, n in enumerate(lens)]
    got = score.continuation_logprobs(v, 2, int(prompt[-1]), conts, [0, 1, 3, 4, 5, 6, 7, 8, 9])
    tol = TOL[s.dtype][0]
    for c, lp in zip(conts, got):
        # every token in one causal pass; the draft part of a longer continuation is at most 64 tokens deep
        full = np.concatenate([prompt, c])
        see = window_ref.context_see(len(full), *window)
        lg = m.logits(full, np.arange(len(full)), see)[len(prompt) - 1:-1]
        want = np.array([ref.logprobs(r)[0][t] for r, t in zip(lg, c)])
        # a logit within tol moves ln sum e^x by at most tol too
        assert np.abs(lp - want).max() <= 2 * tol, (len(c), np.abs(lp - want).max())
    assert v.length(2) == 209
    best, scores = score.choose(v, 2, int(prompt[-1]), conts, [0, 1])
    np.testing.assert_allclose(scores, [lp.sum() for lp in got], atol=2 * tol * 90)
    assert best == int(np.argmax(scores))
    mean = score.choose(v, 2, int(prompt[-1]), conts[:3], [5], per_token=True)[1]
    np.testing.assert_allclose(mean, [lp.mean() for lp in got[:3]], atol=2 * tol)


def test_scoring_refusals(models):
    v, _ = models("f32")
    for bad in (dict(scratch=[]), dict(scratch=[0, 1]), dict(continuations=[[]])):
        kw = dict(dict(continuations=[[1, 2]], scratch=[1, 2]), **bad)
        with pytest.raises(ValueError):
            score.continuation_logprobs(v, 0, 1, kw["continuations"], kw["scratch"])


def test_scoring_refuses_tokens_outside_the_vocabulary(models):
    """The last token of a continuation never goes through the decoder: it is checked like the others."""
    v, _ = models("f32")
    start(v, 0, synth.context_tokens(TINY.vocab, 20, stream=195), 0, 0)
    for bad in ([3, TINY.vocab], [TINY.vocab], [-1], [3, -1], [TINY.vocab, 3], [2 ** 32 + 3], [1.5]):
        for fn in (score.continuation_logprobs, score.choose):
            with pytest.raises(ValueError):
                fn(v, 0, 1, [[4, 5], bad], [1, 2])
    assert v.length(0) == 20
