"""The operators of libtss.so on torch tensors: log probabilities of given
tokens, attention with a sliding window and sinks over a paged KV cache, and
copies of cache pages.

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
    _on_device(q, "q", dev)
    hd = kv.head_dim
    if q.dim() != 3 or q.dtype != pages.dtype or q.shape[2] != hd or q.shape[1] < 1 or q.shape[1] % kv.n_kv_heads:
        raise ValueError("q must be [rows][a multiple of the cache's heads][head_dim] of the cache's type")
    rows, heads, _ = q.shape
    out = torch.empty((rows, heads, hd), dtype=q.dtype, device=dev) if out is None else out
    _on_device(out, "out", dev)
    if out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must be like q")
    for t, name in ((q, "q"), (out, "out")):
        if rows and (t.stride(2) != 1 or t.stride(1) != hd or (rows > 1 and t.stride(0) < heads * hd)):
            raise ValueError(f"a row of {name} must hold its heads one after the other")
    if kv.n_seqs:
        offs = _indices(row_offsets, "row_offsets", (kv.n_seqs + 1,), dev)
        lens = _indices(lengths, "lengths", (kv.n_seqs,), dev)
    else:
        offs = lens = None
    max_rows = rows if max_rows is None else min(max_rows, rows)
    cap = kv.table_stride * PAGE
    max_length = cap if max_length is None else min(max_length, cap)
    if scale is None:
        scale = 0.0                      # the library's default
    elif ctypes.c_float(scale).value == 0:
        raise ValueError("scale must not be 0 in fp32 (None is 1 / sqrt(head_dim))")
    need = abi.tss_window_attn_bytes(kv, heads, rows, max_rows, max_length, sinks, window)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    width = heads * hd
    _call(dev, abi.tss_window_attn, kv, layer, q.data_ptr(), q.stride(0) if rows > 1 else width, heads, offs, lens,
          rows, max_rows, max_length, sinks, window, scale, out.data_ptr(), out.stride(0) if rows > 1 else width,
          ws.data_ptr() if need else None, need)
    return out


def copy_pages(pages, src, dst):
    """pages[:, dst[i]] = pages[:, src[i]] for every i.  src, dst: host lists of page ids; a page may be the source of
    several copies, a destination appears once and is no source."""
    kv = _cache(pages)
    _call(pages.device, abi.tss_copy_pages, kv, src, dst)


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
