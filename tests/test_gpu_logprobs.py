"""Log probabilities of given tokens, entropy and alternatives against plain 64-bit forms: every type, odd sizes and
strides, ties, masked logits, empty rows, infinities and NaN, replays of a captured call, another stream."""
import numpy as np
import pytest
import torch

from paper_2609_26100_amd import ops
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def check(x, tokens, top_k, got, rows=None):
    """Compares with the 64-bit form; x: the logits as the call saw them."""
    V = x.shape[1]
    host = x.double().cpu().numpy()
    tok = None if tokens is None else tokens.cpu().numpy().reshape(len(host), -1)
    g = [None if t is None else t.cpu().numpy() for t in got]
    for r in (range(len(host)) if rows is None else rows):
        o = ref.order(host[r])
        lp, ent = ref.logprobs(host[r])
        tol = ref.logprob_bound(V, lp)
        if np.isnan(ent):
            assert np.isnan(g[2][r])
        else:
            assert abs(g[2][r] - ent) <= ref.entropy_bound(V, lp), (r, g[2][r], ent)

        def same(a, i):
            if np.isfinite(lp[i]):
                assert abs(a - lp[i]) <= tol[i], (r, i, a, lp[i])
            else:
                assert a == lp[i] or (np.isnan(a) and np.isnan(lp[i])), (r, i, a, lp[i])
        if tok is not None:
            place = np.empty(V, np.int64)
            place[o] = np.arange(V)
            for j, t in enumerate(tok[r]):
                a, k = g[0].reshape(len(host), -1)[r, j], g[1].reshape(len(host), -1)[r, j]
                if 0 <= t < V:
                    same(a, t)
                    assert k == place[t], (r, j, t, k, place[t])
                else:
                    assert np.isnan(a) and k == -1
        if top_k:
            np.testing.assert_array_equal(g[4][r], o[:top_k], err_msg=f"row {r}")
            for j in range(top_k):
                same(g[3][r, j], o[j])


def logits(rows, vocab, kind, seed, pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    x = 3 * torch.randn(rows, vocab + pad, generator=g)
    x[:, ::97] += 6
    return x.to(TYPES[kind]).to(DEV)[:, offset:offset + vocab]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,vocab,pad,offset,n,top", [
    (1, 1, 0, 0, 1, 1), (2, 31, 0, 0, 2, 31), (3, 64, 1, 1, 0, 5), (1, 1000, 3, 2, 8, 0), (5, 4096, 0, 0, 1, 32),
    (61, 32000, 0, 0, 1, 20), (6, 32001, 0, 0, 3, 7), (33, 50021, 5, 3, 4, 8), (1, 131072, 0, 0, 1, 32),
    (2, 200003, 1, 1, 1, 1), (300, 777, 0, 0, 1, 2), (1, 16384, 0, 0, 1, 32), (1, 16385, 0, 0, 1, 3),
    (3, 8191, 0, 0, 1, 9), (700, 9001, 0, 0, 2, 4)])
def test_logprobs(kind, rows, vocab, pad, offset, n, top):
    x = logits(rows, vocab, kind, vocab + rows, pad, offset)
    g = torch.Generator().manual_seed(7)
    tok = torch.randint(0, vocab, (rows, n), generator=g, dtype=torch.int32).to(DEV) if n else None
    if n > 1:
        tok[0, 0], tok[-1, -1], tok[0, 1] = vocab, -1, vocab - 1  # pads, the last token
    got = ops.token_logprobs(x, tok, top)
    check(x, tok, top, got, rows=None if rows <= 64 else list(range(0, rows, 29)) + [rows - 1])


def test_tokens_of_one_column():
    x = logits(4, 1003, "f32", 5)
    tok = torch.tensor([0, 5, 1002, -7], dtype=torch.int32, device=DEV)
    got = ops.token_logprobs(x, tok)
    assert got.logprob.shape == got.rank.shape == (4,) and got.top_token is None
    check(x, tok, 0, got)
    alone = ops.token_logprobs(x, None, 3)
    assert alone.logprob is None and alone.rank is None
    check(x, None, 3, alone)
    assert ops.token_logprobs(x[:0], tok[:0], 2).top_token.shape == (0, 2)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("vocab", [40, 5000, 40000])
def test_ties_and_special_rows(kind, vocab):
    """Equal logits (a flat row, few distinct values), signed zeros, masked logits, empty rows, one token left, the
    type's lowest value as a mask, infinities and NaN, values far apart."""
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(14, vocab, generator=g)
    low = torch.finfo(TYPES[kind]).min
    x[0] = 0.25                                        # flat
    x[1] = torch.randint(0, 3, (vocab,), generator=g)  # three values
    x[2] = 0.0
    x[2, ::2] = -0.0
    x[3, torch.rand(vocab, generator=g) < 0.9] = -torch.inf
    x[4] = -torch.inf                                  # nothing left
    x[5] = -torch.inf
    x[5, vocab - 3] = -4.0                             # one token left
    x[6, torch.rand(vocab, generator=g) < 0.9] = low
    x[7] = low
    x[8, vocab // 2] = torch.nan
    x[9, [1, vocab - 1]] = torch.nan
    x[10, 3] = torch.inf
    x[11] = -torch.inf
    x[11, vocab - 2] = torch.nan
    x[12] *= 1e4
    x[13] = torch.arange(vocab) * 1e-3                 # the largest last
    x = x.to(TYPES[kind]).to(DEV)
    tok = torch.randint(0, vocab, (14, 3), generator=g, dtype=torch.int32)
    tok[:, 0] = torch.tensor([vocab - 1, 0, 1, 0, vocab - 1, vocab - 3, 0, 5, vocab // 2, vocab - 1, 3, vocab - 2, 0,
                              vocab - 1])
    tok = tok.to(DEV)
    for top in (0, 1, 32):
        check(x, tok, top, ops.token_logprobs(x, tok, top))


def test_logits_beyond_4_gib():
    rows, vocab = 18000, 131075                  # 4.7 GB, rows that are not aligned
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    x[-40:] = logits(40, vocab, "bf16", 9)
    tok = torch.full((rows, 2), 3, dtype=torch.int32, device=DEV)
    got = ops.token_logprobs(x, tok, 4)
    tail = ops.TokenLogprobs(*(t[-40:] for t in got))
    check(x[-40:], tok[-40:], 4, tail)
    flat = ops.TokenLogprobs(*(t[:2] for t in got))  # all equal: the first tokens, each 1 / vocab
    check(x[:2], tok[:2], 4, flat)


def test_the_same_bits_every_time():
    x = logits(40, 32000, "f32", 11)
    tok = torch.arange(40, dtype=torch.int32, device=DEV)
    a = ops.token_logprobs(x, tok, 20)
    for _ in range(3):
        b = ops.token_logprobs(x, tok, 20)
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_rows_do_not_depend_on_the_batch():
    """Ranks and alternatives of a row are the same alone and among others."""
    x = logits(200, 40000, "bf16", 12)
    all_rows = ops.token_logprobs(x, None, 16)
    for r in (0, 77, 199):
        one = ops.token_logprobs(x[r:r + 1], None, 16)
        assert torch.equal(one.top_token[0], all_rows.top_token[r])


@pytest.mark.parametrize("rows,vocab", [(1, 32000), (3, 150001), (100, 32000)])
def test_captured_and_replayed(rows, vocab):
    x = logits(rows, vocab, "f32", 13)
    tok = torch.zeros(rows, 1, dtype=torch.int32, device=DEV)
    ops.token_logprobs(x, tok, 9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.token_logprobs(x, tok, 9)
    for seed in (21, 22, 23):
        x.copy_(logits(rows, vocab, "f32", seed))
        tok.fill_(seed)
        graph.replay()
        torch.cuda.synchronize()
        eager = ops.token_logprobs(x, tok, 9)
        assert all(torch.equal(p, q) for p, q in zip(got, eager))
    check(x, tok, 9, got, rows=[0, rows - 1])


def test_two_streams_at_once():
    xs = [logits(1, 150001, "f16", s) for s in (31, 32)]
    want = [ops.token_logprobs(x, None, 32) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ops.token_logprobs(xs[i], None, 32))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(p, q) for p, q in zip(r, want[i]) if p is not None)


def test_refusals():
    x = logits(4, 100, "f32", 1)
    tok = torch.zeros(4, dtype=torch.int32, device=DEV)
    for bad in (lambda: ops.token_logprobs(x.t()), lambda: ops.token_logprobs(x[0]),
                lambda: ops.token_logprobs(x.double()), lambda: ops.token_logprobs(x, tok.long()),
                lambda: ops.token_logprobs(x, tok[:3]), lambda: ops.token_logprobs(x, tok.cpu()),
                lambda: ops.token_logprobs(x, None, 33), lambda: ops.token_logprobs(x, None, -1),
                lambda: ops.token_logprobs(x[:, :3], None, 4),
                lambda: ops.token_logprobs(x, torch.zeros(4, 9, dtype=torch.int32, device=DEV)),
                lambda: ops.token_logprobs(x[:1].expand(4, 100)), lambda: ops.token_logprobs(x[:, :0])):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,vocab,pad,offset", [(2, 1000, 0, 0), (1, 1000, 3, 2), (3, 7000, 5, 3), (2, 50021, 1, 1)])
def test_tokens_outside_the_vocabulary(kind, rows, vocab, pad, offset):
    """Pads of any value, inside the last chunk's span too: NaN and -1, and nothing is read for them; the other tokens
    of the row and the alternatives are as without them."""
    x = logits(rows, vocab, kind, vocab, pad, offset)
    pads = [vocab, vocab + 1, vocab + 3, vocab + 1051, 2 ** 31 - 1, -1, -2 ** 31]
    g = torch.Generator().manual_seed(3)
    for first in (0, 3):
        tok = torch.randint(0, vocab, (rows, 8), generator=g, dtype=torch.int32)
        for r in range(rows):
            tok[r, 1:5] = torch.tensor([pads[(first + r + i) % 7] for i in range(4)], dtype=torch.int32)
        tok = tok.to(DEV)
        got = ops.token_logprobs(x, tok, 5)
        check(x, tok, 5, got)
        plain = ops.token_logprobs(x, tok[:, 5:].contiguous(), 5)
        assert torch.equal(got.logprob[:, 5:], plain.logprob) and torch.equal(got.rank[:, 5:], plain.rank)
        assert torch.equal(got.entropy, plain.entropy) and torch.equal(got.top_token, plain.top_token)


@pytest.mark.parametrize("vocab", [40, 5000, 40000])
@pytest.mark.parametrize("kind,size", [(k, s) for s in (1e4, 6e4, 1e5, 1e6, 1e9, 1e10, 1e12, 1e20, 1e30, 3e38)
                                       for k, t in TYPES.items() if s <= torch.finfo(t).max])
def test_rows_at_large_magnitudes(kind, vocab, size):
    """Finite masks and maxima of any size: flat rows, masked rows, rows of which only the first tokens are left (whole
    chunks at the mask's value), maxima far above zero, all of them spread that far."""
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(9, vocab, generator=g)
    noise = x.clone()
    x[0], x[1] = -size, size                           # flat
    x[2, torch.rand(vocab, generator=g) < 0.9] = -size
    x[3, 7:] = -size                                   # only the first are left
    x[4, :vocab - 5] = -size                           # only the last are left
    x[5] = size * (1 - 1e-3 * noise[5].abs().clamp_max(5))
    x[6] = -size * (1 - 1e-3 * noise[6].abs().clamp_max(5))
    x[7] = size * (noise[7] / 8).clamp(-1, 1)
    x[8, vocab // 3] = size                            # one token far ahead
    x = x.to(TYPES[kind]).to(DEV)
    assert torch.isfinite(x).all()
    tok = torch.randint(0, vocab, (9, 3), generator=g, dtype=torch.int32)
    tok[:, 0] = torch.tensor([0, vocab - 1, 5, 3, vocab - 2, 1, 2, 4, vocab // 3])
    tok = tok.to(DEV)
    for top in (0, 9):
        check(x, tok, top, ops.token_logprobs(x, tok, top))
