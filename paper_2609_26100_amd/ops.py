"""The operators of libtss.so on torch tensors: log probabilities of given
tokens, attention with a sliding window and sinks over a paged KV cache, copies of
cache pages; and those of decoding several continuations of one prompt: rows appended
to the cache with the rotation of their positions, attention behind a shared prefix,
the choice of the next beams and the reordering of their cached tokens.

PyTorch only provides the device memory (outputs and workspaces) and the current
stream of the tensors' device, on which every call is enqueued; no call waits.
Arguments that the kernels cannot take are refused with ValueError or TSSError.

A cache is a contiguous tensor [layers][pages][2][kv heads][16 * head_dim] of
float16 or float32 as the verifier lays its pages out: 16 tokens a page, K as
[16][head_dim], V as [4][head_dim][4] (token t at [t // 4, :, t % 4]).
pack_pages and unpack_pages convert.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch

from . import tss as abi

_TYPES = {torch.float32: abi.TSS_T_F32, torch.bfloat16: abi.TSS_T_BF16, torch.float16: abi.TSS_T_F16}
PAGE = 16


class TokenLogprobs(NamedTuple):
    logprob: Optional[torch.Tensor]      # [rows][n] (as tokens), None without tokens
    rank: Optional[torch.Tensor]         # tokens that come before it (0: the greedy token)
    entropy: torch.Tensor                # [rows], nats
    top_logprob: Optional[torch.Tensor]  # [rows][top_k], None for top_k = 0
    top_token: Optional[torch.Tensor]


class BeamSelection(NamedTuple):
    score: torch.Tensor                  # [groups][n] float32, the best first
    parent: torch.Tensor                 # [groups][n] int32: beam of the group that it continues
    token: torch.Tensor                  # [groups][n] int32


def _on_device(t, name, device=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on the GPU")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")


def _indices(t, name, shape, device):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.shape != shape or t.device != device \
            or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


# The current stream's handle without a Stream object around it: with the object,
# a call of 15 us spends 2 of them on it.
_current_stream = torch._C._cuda_getCurrentRawStream


def _call(device, fn, *args):
    """fn on the current stream of the tensors' device, which is the current one during the call."""
    index = device.index
    if torch.cuda.current_device() == index:
        return fn(_current_stream(index), *args)
    with torch.cuda.device(device):
        return fn(_current_stream(index), *args)


def token_logprobs(logits, tokens=None, top_k=0):
    """Log probabilities of given tokens, entropy and the top_k (at most 32) alternatives of each row.

    logits: [rows][vocab] float32, float16 or bfloat16, rows contiguous.  tokens: None, or int32 [rows] or
    [rows][n] with n <= 8 (outside [0, vocab): logprob NaN, rank -1).  Returns TokenLogprobs; ties go to the lower
    token, see tss_token_logprobs for infinities and NaN."""
    _on_device(logits, "logits")
    dev = logits.device
    if logits.dim() != 2 or logits.dtype not in _TYPES:
        raise ValueError("logits must be [rows][vocab] of float32, float16 or bfloat16")
    rows, vocab = logits.shape
    if vocab < 1 or (rows and vocab > 1 and logits.stride(1) != 1) or (rows > 1 and logits.stride(0) < vocab):
        raise ValueError("rows of logits must be contiguous and must not overlap")
    n, tok = 0, None
    if tokens is not None:
        if not isinstance(tokens, torch.Tensor) or tokens.dim() not in (1, 2) or tokens.shape[0] != rows:
            raise ValueError("tokens must be [rows] or [rows][n]")
        n = 1 if tokens.dim() == 1 else tokens.shape[1]
        tok = _indices(tokens, "tokens", tokens.shape, dev)
    if not 0 <= top_k <= min(vocab, abi.TSS_LOGPROBS_MAX_TOP) or n > abi.TSS_LOGPROBS_MAX_TOKENS:
        raise ValueError("at most 8 tokens a row and min(32, vocab) alternatives")
    f32, i32, empty = torch.float32, torch.int32, torch.empty
    ent = empty(rows, dtype=f32, device=dev)
    lp = rank = top_lp = top_tok = None
    if tokens is not None:
        lp, rank = empty(tokens.shape, dtype=f32, device=dev), empty(tokens.shape, dtype=i32, device=dev)
    if top_k:
        top_lp, top_tok = empty((rows, top_k), dtype=f32, device=dev), empty((rows, top_k), dtype=i32, device=dev)
    need = abi.tss_token_logprobs_bytes(rows, vocab, n, top_k)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    stride = logits.stride(0) if rows > 1 else vocab
    _call(dev, abi.tss_token_logprobs, logits.data_ptr(), _TYPES[logits.dtype], stride, rows, vocab,
          tok if n else None, n, top_k, lp.data_ptr() if n else None, rank.data_ptr() if n else None, ent.data_ptr(),
          top_lp.data_ptr() if top_k else None, top_tok.data_ptr() if top_k else None,
          ws.data_ptr() if need else None, need)
    return TokenLogprobs(lp, rank, ent, top_lp, top_tok)


def _cache(pages, page_table=None):
    _on_device(pages, "pages")
    if pages.dim() != 5 or pages.dtype not in (torch.float16, torch.float32) or pages.shape[2] != 2 \
            or pages.shape[4] not in (PAGE * 64, PAGE * 128) or not pages.is_contiguous():
        raise ValueError("pages must be a contiguous float16 or float32 tensor [layers][pages][2][heads][16 * 64 or 128]")
    L, P, _, H, e = pages.shape
    kv = abi.tss_paged_kv(pages.data_ptr(), None, L, P, H, e // PAGE, _TYPES[pages.dtype], 0, 0)
    if page_table is not None:
        if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
            raise ValueError("page_table must be [sequences][pages of a sequence]")
        kv.page_table = _indices(page_table, "page_table", page_table.shape, pages.device)
        kv.n_seqs, kv.table_stride = page_table.shape
    return kv


def _by_heads(t, name, shape):
    """Refuses a tensor of this shape [rows][heads][head_dim] whose rows do not hold their heads one after the other; the
    rows' stride."""
    rows, heads, hd = shape
    row, head, one = t.stride()
    if rows and (one != 1 or (head != hd and heads > 1) or (row < heads * hd and rows > 1)):
        raise ValueError(f"a row of {name} must hold its heads one after the other")
    return row if rows > 1 else heads * hd


def _queries(kv, q, pages, scale, out):
    """Checks of an attention call's q, out and scale: (rows, heads, out, strides of q and out, scale)."""
    dev = pages.device
    _on_device(q, "q", dev)
    shape, dtype = q.shape, q.dtype
    if len(shape) != 3 or dtype != pages.dtype or shape[2] != kv.head_dim or shape[1] < 1 or shape[1] % kv.n_kv_heads:
        raise ValueError("q must be [rows][a multiple of the cache's heads][head_dim] of the cache's type")
    if out is None:
        out, out_stride = torch.empty(shape, dtype=dtype, device=dev), shape[1] * shape[2]
    else:
        _on_device(out, "out", dev)
        if out.shape != shape or out.dtype != dtype:
            raise ValueError("out must be like q")
        out_stride = _by_heads(out, "out", shape)
    if scale is None:
        scale = 0.0                      # the library's default
    elif ctypes.c_float(scale).value == 0:
        raise ValueError("scale must not be 0 in fp32 (None is 1 / sqrt(head_dim))")
    return shape[0], shape[1], out, _by_heads(q, "q", shape), out_stride, scale


def _sequences(kv, row_offsets, lengths, rows, max_rows, max_length, dev):
    """(row_offsets, lengths, max_rows, max_length) as the library takes them."""
    offs = lens = None
    if kv.n_seqs:
        offs = _indices(row_offsets, "row_offsets", (kv.n_seqs + 1,), dev)
        lens = _indices(lengths, "lengths", (kv.n_seqs,), dev)
    cap = kv.table_stride * PAGE
    return (offs, lens, rows if max_rows is None else min(max_rows, rows),
            cap if max_length is None else min(max_length, cap))


def window_attention(q, pages, page_table, row_offsets, lengths, sinks=0, window=0, layer=0, scale=None,
                     max_rows=None, max_length=None, out=None):
    """Attention of one layer: row i of a sequence of r rows is the token at p = length - r + i and sees token t
    when t <= p and (t < sinks or t > p - window); window 0 sees every t <= p.

    q: [rows][heads][head_dim] of the cache's type, heads a multiple of the cache's; page_table: int32
    [sequences][n]; row_offsets: int32 [sequences + 1], increasing from 0; lengths: int32 [sequences], cached
    tokens with the queries' own.  max_rows and max_length: upper bounds of a sequence's rows and length (without
    them all of q's rows and the page table's tokens; tighter bounds launch less).  scale: factor of q k, above 0;
    None for 1 / sqrt(head_dim).  out: like q, may be q, otherwise shares no element with it.  Rows of out behind the
    last sequence are left as they were."""
    kv = _cache(pages, page_table)
    dev = pages.device
    rows, heads, out, q_stride, out_stride, scale = _queries(kv, q, pages, scale, out)
    offs, lens, max_rows, max_length = _sequences(kv, row_offsets, lengths, rows, max_rows, max_length, dev)
    need = abi.tss_window_attn_bytes(kv, heads, rows, max_rows, max_length, sinks, window)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(dev, abi.tss_window_attn, kv, layer, q.data_ptr(), q_stride, heads, offs, lens, rows, max_rows, max_length,
          sinks, window, scale, out.data_ptr(), out_stride, ws.data_ptr() if need else None, need)
    return out


def copy_pages(pages, src, dst):
    """pages[:, dst[i]] = pages[:, src[i]] for every i.  src, dst: host lists of page ids; a page may be the source of
    several copies, a destination appears once and is no source."""
    kv = _cache(pages)
    _call(pages.device, abi.tss_copy_pages, kv, src, dst)


@functools.lru_cache(maxsize=64)
def _frequencies(base, head_dim):
    """base^(-2j / head_dim) for the head's pairs, as the library takes them."""
    half = head_dim // 2
    return (ctypes.c_double * half)(*(float(base) ** (-2.0 * j / head_dim) for j in range(half)))


def _rotation(rope, head_dim):
    """append_kv's rope as the library takes it."""
    if rope is None:
        return None
    if not hasattr(rope, "__len__") or getattr(rope, "ndim", 1) == 0:      # a number, or an array of one without axes
        rope = float(rope)
        if not 0 < rope < float("inf"):
            raise ValueError("the rotation's base must be positive and finite")
        try:
            return _frequencies(rope, head_dim)
        except OverflowError:
            raise ValueError("the rotation's base is too small: its frequencies exceed float64") from None
    freq = [float(x) for x in rope]
    if len(freq) != head_dim // 2:
        raise ValueError("rope must have head_dim / 2 frequencies")
    return (ctypes.c_double * len(freq))(*freq)


def append_kv(q, k, v, pages, page_table, row_offsets, lengths, positions=None, rope=10000.0, layer=0, max_rows=None,
              out=None):
    """Appends rows to one layer of the cache, rotated to their positions, and returns their rotated queries: row i of
    a sequence of r rows is the token of slot lengths - r + i (rows and lengths as window_attention has them).

    q: [rows][any heads][head_dim] (None: keys and values alone, returns None), k, v: [rows][the cache's
    heads][head_dim], all of one type, float32, float16 or bfloat16; rows may be apart, as parts of one projection's
    output are.  positions: int32 [rows], for rows whose position is not their slot (a tree's nodes, which the attentions
    here do not keep from seeing their siblings).  rope: the rotation's base, or its head_dim / 2 frequencies (host
    numbers), or None for no rotation.  max_rows: upper bound of a sequence's rows.  out: the rotated queries, of the
    cache's type; may be q, otherwise shares no element with an input.  Rows behind the last sequence and before token 0
    are left as they were."""
    kv = _cache(pages, page_table)
    dev, hd = pages.device, kv.head_dim
    _on_device(k, "k", dev)
    _on_device(v, "v", dev)
    shape, dtype = k.shape, k.dtype
    if len(shape) != 3 or shape[1] != kv.n_kv_heads or shape[2] != hd or dtype not in _TYPES or v.shape != shape \
            or v.dtype != dtype:
        raise ValueError("k and v must be [rows][the cache's heads][head_dim] of one type")
    rows, heads = shape[0], 0
    q_at = q_out = None
    q_stride = out_stride = 0
    if q is None:
        out = None
    else:
        _on_device(q, "q", dev)
        q_shape = q.shape
        if len(q_shape) != 3 or q_shape[0] != rows or q_shape[2] != hd or q.dtype != dtype:
            raise ValueError("q must be [rows][heads][head_dim] of k's type and number of rows")
        heads = q_shape[1]
        if out is None:
            out, out_stride = torch.empty(q_shape, dtype=pages.dtype, device=dev), heads * hd
        else:
            _on_device(out, "out", dev)
            if out.shape != q_shape or out.dtype != pages.dtype:
                raise ValueError("out must be like q, of the cache's type")
            out_stride = _by_heads(out, "out", q_shape)
        if heads:
            q_at, q_out, q_stride = q.data_ptr(), out.data_ptr(), _by_heads(q, "q", q_shape)
    offs, lens, max_rows, _ = _sequences(kv, row_offsets, lengths, rows, max_rows, None, dev)
    pos = None if positions is None else _indices(positions, "positions", (rows,), dev)
    freq = _rotation(rope, hd)
    _call(dev, abi.tss_append_kv, kv, layer, q_at, q_stride, heads, k.data_ptr(), _by_heads(k, "k", shape), v.data_ptr(),
          _by_heads(v, "v", shape), _TYPES[dtype], offs, lens, pos, rows, max_rows, freq, q_out, out_stride)
    return out


def prefix_attention(q, pages, page_table, row_offsets, lengths, shared, group_offsets=None, layer=0, scale=None,
                     max_rows=None, max_length=None, max_shared=None, max_group_rows=None, out=None):
    """Attention of one layer for sequences that share a prefix: what window_attention gives without a window, but the
    pages that a group of sequences has in common are read once for all of its rows.

    shared: int32 [groups], how many first entries of the page tables of a group's sequences name the same pages.
    group_offsets: int32 [groups + 1], a group's first sequences; None for one group of all (then shared has one entry).
    max_shared and max_group_rows: upper bounds of a group's shared pages and rows (without them the page table's and
    all of q's).  The work is cut up by the bounds, so tight ones, max_rows and max_length too, take less time.  The
    other arguments are window_attention's."""
    kv = _cache(pages, page_table)
    dev = pages.device
    rows, heads, out, q_stride, out_stride, scale = _queries(kv, q, pages, scale, out)
    offs, lens, max_rows, max_length = _sequences(kv, row_offsets, lengths, rows, max_rows, max_length, dev)
    if not isinstance(shared, torch.Tensor) or shared.dim() != 1:
        raise ValueError("shared must be an int32 tensor [groups]")
    groups = shared.shape[0]
    shared = _indices(shared, "shared", shared.shape, dev)
    if group_offsets is not None:
        group_offsets = _indices(group_offsets, "group_offsets", (groups + 1,), dev)
    elif groups != 1:
        raise ValueError("several groups need group_offsets")
    max_shared = kv.table_stride if max_shared is None else min(max_shared, kv.table_stride)
    max_group_rows = rows if max_group_rows is None else min(max_group_rows, rows)
    need = abi.tss_prefix_attn_bytes(kv, heads, rows, max_rows, max_length, groups, max_group_rows, max_shared)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(dev, abi.tss_prefix_attn, kv, layer, q.data_ptr(), q_stride, heads, offs, lens, rows, max_rows, max_length,
          group_offsets, shared, groups, max_group_rows, max_shared, scale, out.data_ptr(), out_stride,
          ws.data_ptr() if need else None, need)
    return out


def beam_select(logits, scores, n, ended=None, end_token=None):
    """The n best continuations of each group of beams, by scores[beam] + log probability of the token.

    logits: [groups * beams][vocab] float32, float16 or bfloat16, rows contiguous.  scores: float32 [groups][beams], at
    most 32 beams.  ended: int32 [groups][beams], not 0 for a beam that has ended: its one candidate is end_token, with its
    score as it is.  Returns BeamSelection, each [groups][n], n <= min(64, beams * vocab); ties go to the lower beam,
    then to the lower token; see tss_beam_select for what is worth -inf."""
    _on_device(logits, "logits")
    dev = logits.device
    if logits.dim() != 2 or logits.dtype not in _TYPES:
        raise ValueError("logits must be [groups * beams][vocab] of float32, float16 or bfloat16")
    rows, vocab = logits.shape
    if vocab < 1 or (rows and vocab > 1 and logits.stride(1) != 1) or (rows > 1 and logits.stride(0) < vocab):
        raise ValueError("rows of logits must be contiguous and must not overlap")
    if not isinstance(scores, torch.Tensor) or scores.dim() != 2 or scores.dtype != torch.float32 \
            or scores.device != dev or not scores.is_contiguous() or scores.numel() != rows:
        raise ValueError("scores must be a contiguous float32 tensor [groups][beams], a score for each row of logits")
    groups, beams = scores.shape
    at = None
    if ended is not None:
        if end_token is None or not 0 <= end_token < vocab:
            raise ValueError("beams that have ended need an end_token of the vocabulary")
        at = _indices(ended, "ended", scores.shape, dev)
    if not 1 <= beams <= abi.TSS_BEAMS_MAX or not 1 <= n <= min(abi.TSS_BEAMS_MAX_N, beams * vocab):
        raise ValueError("at most 32 beams, and from 1 to min(64, beams * vocab) continuations")
    i32 = torch.int32
    score = torch.empty((groups, n), dtype=torch.float32, device=dev)
    parent, token = torch.empty((groups, n), dtype=i32, device=dev), torch.empty((groups, n), dtype=i32, device=dev)
    need = abi.tss_beam_select_bytes(groups, beams, vocab, n)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(dev, abi.tss_beam_select, logits.data_ptr(), _TYPES[logits.dtype], logits.stride(0) if rows > 1 else vocab,
          groups, beams, vocab, scores.data_ptr(), at, end_token if at else 0, n, score.data_ptr(), parent.data_ptr(),
          token.data_ptr(), ws.data_ptr() if need else None, need)
    return BeamSelection(score, parent, token)


def reorder_pages(pages, page_table, parents, lengths, shared=None, max_own=None):
    """Sequence g * beams + b becomes what sequence g * beams + parents[g][b] was, in every layer and in place, all of a
    group at once.

    parents: int32 [groups][beams], at most 32 beams; page_table has groups * beams sequences.  lengths: int32 [groups *
    beams], tokens of each sequence before the call.  shared: int32 [groups], first pages that the group's sequences have
    in common, which stay (None: no page); the pages behind them must be each sequence's own.  max_own: upper bound
    of the tokens behind the shared pages (None: the page table's; a tighter bound launches less).  The caller moves
    its own lengths, lengths[parents]."""
    kv = _cache(pages, page_table)
    dev = pages.device
    if not isinstance(parents, torch.Tensor) or parents.dim() != 2 or parents.numel() != kv.n_seqs:
        raise ValueError("parents must be [groups][beams], an entry for each sequence of the page table")
    groups, beams = parents.shape
    if not 1 <= beams <= abi.TSS_BEAMS_MAX:
        raise ValueError("from 1 to 32 beams")
    par = _indices(parents, "parents", parents.shape, dev)
    lens = _indices(lengths, "lengths", (kv.n_seqs,), dev)
    at = None if shared is None else _indices(shared, "shared", (groups,), dev)
    cap = kv.table_stride * PAGE
    _call(dev, abi.tss_reorder_pages, kv, par, beams, lens, at, cap if max_own is None else min(max_own, cap))


def pack_pages(k, v):
    """Cache pages [pages][2][heads][16 * head_dim] of contiguous k and v [tokens][heads][head_dim]; the last page is
    filled up with zeros."""
    n, heads, hd = k.shape
    full = -(-n // PAGE) * PAGE
    kv = torch.zeros((2, full, heads, hd), dtype=k.dtype, device=k.device)
    kv[0, :n], kv[1, :n] = k, v
    kp = kv[0].reshape(-1, PAGE, heads, hd).transpose(1, 2).reshape(-1, heads, PAGE * hd)
    vp = kv[1].reshape(-1, 4, 4, heads, hd).permute(0, 3, 1, 4, 2).reshape(-1, heads, PAGE * hd)
    return torch.stack((kp, vp), 1)


def unpack_pages(pages):
    """k and v [tokens][heads][head_dim] of pages [pages][2][heads][16 * head_dim]."""
    n, _, heads, e = pages.shape
    hd = e // PAGE
    k = pages[:, 0].reshape(n, heads, PAGE, hd).transpose(1, 2).reshape(n * PAGE, heads, hd)
    v = pages[:, 1].reshape(n, heads, 4, hd, 4).permute(0, 2, 4, 1, 3).reshape(n * PAGE, heads, hd)
    return k, v
