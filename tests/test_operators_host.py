"""What the operators refuse, on the CPU: every check comes before any device work, so the addresses need not exist."""
import ctypes
import types

import numpy as np
import pytest
import torch

from paper_2609_26100_amd import decode, ops, score
from paper_2609_26100_amd import tss as abi

P = 0x10000  # a device address that no check touches


def logprobs(**kw):
    a = dict(logits=P, type=abi.TSS_T_F32, row_stride=100, rows=2, vocab=100, tokens=P, n_tokens=1, top_k=5, logprob=P,
             rank=P, entropy=P, top_logprob=P, top_token=P, workspace=P, workspace_bytes=1 << 30)
    a.update(kw)
    abi.tss_token_logprobs(None, **a)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(type=-1), dict(rows=-1), dict(vocab=0), dict(row_stride=99), dict(n_tokens=9),
    dict(n_tokens=-1), dict(top_k=33), dict(top_k=-1), dict(vocab=4, top_k=5), dict(logits=None), dict(tokens=None),
    dict(logits=P + 2), dict(type=abi.TSS_T_F16, logits=P + 1)])
def test_logprobs_refuses(bad):
    with pytest.raises(abi.TSSError) as e:
        logprobs(**bad)
    assert e.value.status == abi.TSS_EINVAL and "tss_token_logprobs" in str(e.value)


def test_logprobs_workspace():
    need = abi.tss_token_logprobs_bytes(1, 1 << 20, 1, 32)
    if need:
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
            with pytest.raises(abi.TSSError) as e:
                logprobs(**dict(dict(rows=1, vocab=1 << 20, row_stride=1 << 20, top_k=32), **bad))
            assert e.value.status == abi.TSS_ENOSPACE
    logprobs(rows=0)                       # nothing to do
    logprobs(rows=0, logits=None, tokens=None)
    for bad in ((-1, 100, 1, 1), (1, 0, 1, 1), (1, 100, 9, 1), (1, 100, 1, 33), (1, 4, 0, 5)):
        assert abi.tss_token_logprobs_bytes(*bad) == 0


def cache(**kw):
    kv = abi.tss_paged_kv(P, P, 2, 8, 4, 64, abi.TSS_T_F16, 2, 4)
    for k, v in kw.items():
        setattr(kv, k, v)
    return kv


def window(kv=None, **kw):
    a = dict(layer=0, q=P, q_stride=512, n_q_heads=8, row_offsets=P, lengths=P, rows=4, max_rows=4, max_length=64,
             sinks=1, window=16, scale=0.0, out=P, out_stride=512, workspace=P, workspace_bytes=1 << 40)
    a.update(kw)
    abi.tss_window_attn(None, kv or cache(), **a)


@pytest.mark.parametrize("bad", [
    dict(layer=2), dict(layer=-1), dict(q_stride=511), dict(q_stride=504), dict(q_stride=516), dict(out_stride=8),
    dict(n_q_heads=6), dict(n_q_heads=0), dict(rows=-1), dict(max_rows=-1), dict(max_length=-1), dict(sinks=-1),
    dict(window=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None),
    dict(out=None), dict(row_offsets=None), dict(lengths=None), dict(q=P + 8), dict(out=P + 4)])
def test_window_refuses(bad):
    with pytest.raises(abi.TSSError) as e:
        window(**bad)
    assert e.value.status == abi.TSS_EINVAL and "tss_window_attn" in str(e.value)


@pytest.mark.parametrize("bad", [
    dict(pages=None), dict(type=abi.TSS_T_BF16), dict(type=7), dict(head_dim=96), dict(n_layers=0), dict(n_pages=0),
    dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(pages=P + 8)])
def test_cache_refused(bad):
    for call in (window, lambda kv: abi.tss_copy_pages(None, kv, [0], [1])):
        with pytest.raises(abi.TSSError) as e:
            call(cache(**bad))
        assert e.value.status == abi.TSS_EINVAL


def test_window_table_and_workspace():
    for bad in (dict(page_table=None), dict(n_seqs=-1), dict(table_stride=0)):
        with pytest.raises(abi.TSSError):
            window(cache(**bad))
    kv = cache(n_pages=1 << 16, table_stride=1 << 14, n_seqs=1)
    big = dict(rows=1, max_rows=1, max_length=1 << 18, window=0)
    need = abi.tss_window_attn_bytes(kv, 8, 1, 1, 1 << 18, 1, 0)
    if need:
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
            with pytest.raises(abi.TSSError) as e:
                window(kv, **big, **bad)
            assert e.value.status == abi.TSS_ENOSPACE
    for nothing in (dict(rows=0), dict(max_rows=0)):
        window(**nothing, q=None, out=None)
    window(cache(n_seqs=0), row_offsets=None, lengths=None)
    assert abi.tss_window_attn_bytes(cache(head_dim=96), 8, 4, 4, 64, 1, 16) == 0
    assert abi.tss_window_attn_bytes(cache(), 7, 4, 4, 64, 1, 16) == 0


@pytest.mark.parametrize("src,dst", [([0], [8]), ([8], [0]), ([-1], [0]), ([0], [-1]), ([0, 1], [2, 2]), ([0], [0]),
                                     ([0, 1], [1, 2]), ([0, 2], [1, 0])])
def test_copy_refuses(src, dst):
    with pytest.raises(abi.TSSError) as e:
        abi.tss_copy_pages(None, cache(), src, dst)
    assert e.value.status == abi.TSS_EINVAL


def test_copy_lists():
    abi.tss_copy_pages(None, cache(), [], [])
    with pytest.raises(ValueError):
        abi.tss_copy_pages(None, cache(), [0, 1], [2])
    L = abi.lib()
    assert L.tss_copy_pages(None, ctypes.byref(cache()), None, None, 1) == abi.TSS_EINVAL
    assert L.tss_copy_pages(None, ctypes.byref(cache()), P, P, -1) == abi.TSS_EINVAL
    assert L.tss_copy_pages(None, None, P, P, 0) == abi.TSS_EINVAL


def test_tensors_off_the_gpu_are_refused():
    x = torch.zeros(2, 10)
    pages = torch.zeros(1, 2, 2, 1, 16 * 64)
    with pytest.raises(ValueError):
        ops.token_logprobs(x)
    with pytest.raises(ValueError):
        ops.copy_pages(pages, [0], [1])
    with pytest.raises(ValueError):
        ops.window_attention(torch.zeros(1, 1, 64), pages, None, None, None)


@pytest.mark.parametrize("n,heads,hd", [(1, 1, 64), (16, 2, 128), (37, 3, 64)])
def test_pages_and_back(n, heads, hd):
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(n, heads, hd, generator=g).half() for _ in range(2))
    p = ops.pack_pages(k, v)
    assert p.shape == (-(-n // 16), 2, heads, 16 * hd)
    t, d = n - 1, hd - 3  # one element where the layout puts it
    assert p[t // 16, 0, heads - 1].reshape(16, hd)[t % 16, d] == k[t, heads - 1, d]
    assert p[t // 16, 1, heads - 1].reshape(4, hd, 4)[t % 16 // 4, d, t % 4] == v[t, heads - 1, d]
    k2, v2 = ops.unpack_pages(p)
    assert torch.equal(k2[:n], k) and torch.equal(v2[:n], v) and not k2[n:].any() and not v2[n:].any()


def test_message_names_the_last_refusal():
    with pytest.raises(abi.TSSError) as e:
        logprobs(top_k=40)
    assert abi.tss_last_error(None) in str(e.value) and "top_k" in abi.tss_last_error(None)


def test_a_score_of_nan_is_not_chosen(monkeypatch):
    scores = [[float("nan")], [-3.0, -1.0], [-2.0, -1.5], [float("nan"), 0.0]]
    monkeypatch.setattr(score, "continuation_logprobs", lambda *a: [np.asarray(s, np.float32) for s in scores])
    assert score.choose(None, 0, 1, scores, [1])[0] == 2
    assert score.choose(None, 0, 1, scores, [1], per_token=True)[0] == 2


@pytest.mark.parametrize("far", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, -2 ** 31 - 1, -2 ** 32 + 5])
def test_whole_numbers_beyond_32_bits_are_refused(far):
    """None of them is cut off to another one on its way to the library."""
    for name in ("type", "rows", "vocab", "n_tokens", "top_k"):
        with pytest.raises(ValueError):
            logprobs(**{name: far})
    for name in ("layer", "n_q_heads", "rows", "max_rows", "max_length", "sinks", "window"):
        with pytest.raises(ValueError):
            window(**{name: far})
    for i in range(4):
        with pytest.raises(ValueError):
            abi.tss_token_logprobs_bytes(*[far if j == i else 1 for j in range(4)])
    for i in range(6):
        with pytest.raises(ValueError):
            abi.tss_window_attn_bytes(cache(), *[far if j == i else 4 for j in range(6)])
    for call in (lambda: abi.tss_set_window(None, far, 0, 64), lambda: abi.tss_set_window(None, 0, far, 64),
                 lambda: abi.tss_set_window(None, 0, 0, far), lambda: abi.tss_seq_fork(None, far, [1], 0),
                 lambda: abi.tss_seq_fork(None, 0, [1], far), lambda: abi.tss_seq_fork(None, 0, [far], 0),
                 lambda: abi.tss_get_logprobs(None, far), lambda: abi.tss_get_logprobs(None, 1, None, far),
                 lambda: abi.tss_get_logprobs(None, 1, [far]), lambda: abi.tss_get_logprobs(None, 1, [[1, far]])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("pages", [[2 ** 32 + 3], np.array([2 ** 32 + 3]), np.array([3 + 2 ** 32], np.uint64), [1.5],
                                   np.array([1.5]), [float("nan")], [np.int64(2 ** 32 + 3)], [2 ** 70], (2 ** 31,)])
def test_lists_whose_numbers_would_change_are_refused(pages):
    for src, dst in ((pages, [2]), ([2], pages)):
        with pytest.raises(ValueError):
            abi.tss_copy_pages(None, cache(), src, dst)


def test_lists_of_every_kind():
    want = [1, 2, 1 << 30]
    for a in (want, tuple(want), np.array(want), np.array(want, np.uint32), np.array(want, np.int32), np.array(want, float),
              [float(x) for x in want], torch.tensor(want), np.array([want, want]).T[:, 0], [np.int64(x) for x in want]):
        got = abi._int32s(a, "a")
        assert got.dtype == np.int32 and got.tolist() == want and got.flags["C_CONTIGUOUS"]
    assert abi._int32s([[1, 2], [3, 4]], "a").tolist() == [[1, 2], [3, 4]]
    assert abi._int32s([], "a").size == 0 and abi._int32s(np.zeros(0), "a").size == 0


class OneWayVerifier:
    """Answers token 1 to everything and counts the steps that it commits."""

    def __init__(self, vocab=100):
        self.cfg, self.steps = types.SimpleNamespace(vocab=vocab), 0

    def verify(self, seq, tokens, parent=None, mask=None, commit=False):
        self.steps += commit
        return 0, 1

    def logprobs(self, n_nodes, tokens=None, top_k=0):
        return (np.full(n_nodes, -1, np.float32), np.zeros(n_nodes, np.int32), np.zeros(n_nodes, np.float32),
                np.zeros((n_nodes, top_k), np.float32) if top_k else None,
                np.zeros((n_nodes, top_k), np.int32) if top_k else None)


def decodes(v, max_new, logprobs):
    yield lambda: decode.autoregressive_decode(v, 0, 3, max_new, logprobs=logprobs)
    yield lambda: decode.speculative_decode(v, 0, 3, max_new, lambda root, pos: ([root, 5], None), logprobs=logprobs)


@pytest.mark.parametrize("k,vocab", [(33, 100), (-1, 100), (5, 4)])
def test_decoding_refuses_numbers_of_alternatives_before_a_step(k, vocab):
    v = OneWayVerifier(vocab)
    for run in decodes(v, 4, k):
        with pytest.raises(ValueError):
            run()
    assert v.steps == 0


@pytest.mark.parametrize("k", [0, 3])
def test_decoding_no_token_with_log_probabilities(k):
    for n in (0, 2):
        for run in decodes(OneWayVerifier(), n, k):
            r = run()
            assert len(r.tokens) == n
            assert [x.shape for x in (r.logprobs.logprob, r.logprobs.entropy, r.logprobs.top_logprob,
                                      r.logprobs.top_token)] == [(n,), (n,), (n, k), (n, k)]
            assert [x.dtype for x in (r.logprobs.logprob, r.logprobs.top_logprob, r.logprobs.top_token)] == [
                np.float32, np.float32, np.int32]
    assert all(run().logprobs is None for run in decodes(OneWayVerifier(), 0, None))


def test_scale_whose_power_of_two_overflows_is_refused():
    """A factor of finite scores that is finite itself, but not in powers of two."""
    for scale in (2.4e38, 3.4e38):
        with pytest.raises(abi.TSSError) as e:
            window(scale=scale)
        assert e.value.status == abi.TSS_EINVAL and "scale" in str(e.value)


def test_sizes_of_every_whole_type():
    """A short type beside a longer number is no reason to refuse, a fraction is one."""
    for t in (int, np.uint8, np.int16, np.int64, np.uint64):
        assert abi.tss_token_logprobs_bytes(t(3), 40000, t(1), t(5)) == abi.tss_token_logprobs_bytes(3, 40000, 1, 5) > 0
        assert abi.tss_window_attn_bytes(cache(), t(8), t(4), t(4), 1024, t(4), t(100)) == 0
    for bad in (1.0, np.float32(2), None, "4"):
        with pytest.raises(ValueError):
            abi.tss_token_logprobs_bytes(bad, 40000, 1, 5)


@pytest.mark.parametrize("k", [1.5, float("nan"), "3"])
def test_decoding_refuses_what_is_no_number_of_alternatives(k):
    v = OneWayVerifier()
    for run in decodes(v, 4, k):
        with pytest.raises(ValueError):
            run()
    assert v.steps == 0
    assert decode.autoregressive_decode(v, 0, 3, 2, logprobs=2.0).logprobs.top_token.shape == (2, 2)
