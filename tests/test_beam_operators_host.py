"""What the operators of several continuations refuse, on the CPU: every check comes before any device work."""
import ctypes

import pytest
import torch

from paper_2609_26100_amd import ops
from paper_2609_26100_amd import tss as abi

P = 0x10000  # a device address that no check touches
FREQ = (ctypes.c_double * 64)(*[1.0] * 64)


def cache(**kw):
    kv = abi.tss_paged_kv(P, P, 2, 8, 4, 64, abi.TSS_T_F16, 2, 4)
    for k, v in kw.items():
        setattr(kv, k, v)
    return kv


def append(kv=None, **kw):
    a = dict(layer=0, q=P, q_stride=512, n_q_heads=8, k=P, k_stride=256, v=P, v_stride=256, type=abi.TSS_T_F32,
             row_offsets=P, lengths=P, positions=None, rows=4, max_rows=4, inv_freq=FREQ, q_out=P, q_out_stride=512)
    a.update(kw)
    abi.tss_append_kv(None, kv or cache(), **a)


def prefix(kv=None, **kw):
    a = dict(layer=0, q=P, q_stride=512, n_q_heads=8, row_offsets=P, lengths=P, rows=4, max_rows=4, max_length=64,
             group_offsets=P, shared=P, n_groups=1, max_group_rows=4, max_shared=2, scale=0.0, out=P, out_stride=512,
             workspace=P, workspace_bytes=1 << 40)
    a.update(kw)
    abi.tss_prefix_attn(None, kv or cache(), **a)


def beams(**kw):
    a = dict(logits=P, type=abi.TSS_T_F32, row_stride=100, n_groups=2, n_beams=3, vocab=100, scores=P, ended=P,
             end_token=2, n=6, score=P, parent=P, token=P, workspace=P, workspace_bytes=1 << 30)
    a.update(kw)
    abi.tss_beam_select(None, **a)


def reorder(kv=None, **kw):
    a = dict(parents=P, n_beams=2, lengths=P, shared=P, max_own=30)
    a.update(kw)
    abi.tss_reorder_pages(None, kv or cache(), **a)


def refused(call, status, name, *args, **kw):
    with pytest.raises(abi.TSSError) as e:
        call(*args, **kw)
    assert e.value.status == status and name in str(e.value)


@pytest.mark.parametrize("bad", [
    dict(layer=2), dict(layer=-1), dict(type=3), dict(type=-1), dict(q_stride=504), dict(q_stride=516),
    dict(k_stride=248), dict(k_stride=260), dict(v_stride=0), dict(v_stride=300), dict(q_out_stride=508),
    dict(n_q_heads=-1), dict(n_q_heads=65536), dict(rows=-1), dict(max_rows=-1), dict(q=None), dict(k=None),
    dict(v=None), dict(q_out=None), dict(row_offsets=None), dict(lengths=None), dict(q=P + 8), dict(k=P + 4),
    dict(v=P + 2), dict(q_out=P + 8), dict(inv_freq=(ctypes.c_double * 64)(*[float("inf")] * 64)),
    dict(inv_freq=(ctypes.c_double * 64)(*[-1.1e6] * 64)),
    dict(inv_freq=(ctypes.c_double * 64)(*([1.0] * 31 + [float("nan")] + [1.0] * 32)))])
def test_append_refuses(bad):
    refused(append, abi.TSS_EINVAL, "tss_append_kv", **bad)


def test_append_of_nothing():
    append(rows=0, k=None, v=None, q=None)
    append(max_rows=0)
    append(cache(n_seqs=0), row_offsets=None, lengths=None)


@pytest.mark.parametrize("bad", [
    dict(layer=2), dict(layer=-1), dict(q_stride=511), dict(q_stride=504), dict(q_stride=516), dict(out_stride=8),
    dict(n_q_heads=6), dict(n_q_heads=0), dict(rows=-1), dict(max_rows=-1), dict(max_length=-1), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None), dict(row_offsets=None),
    dict(lengths=None), dict(q=P + 8), dict(out=P + 4), dict(n_groups=-1), dict(max_group_rows=-1),
    dict(max_shared=-1), dict(shared=None), dict(group_offsets=None, n_groups=2), dict(n_groups=65536)])
def test_prefix_refuses(bad):
    refused(prefix, abi.TSS_EINVAL, "tss_prefix_attn", **bad)


def test_prefix_of_nothing_and_workspace():
    for nothing in (dict(rows=0), dict(max_rows=0)):
        prefix(**nothing, q=None, out=None)
    prefix(cache(n_seqs=0), row_offsets=None, lengths=None)
    kv = cache(n_pages=1 << 16, table_stride=1 << 12, n_seqs=8)
    sizes = dict(rows=8, max_rows=1, max_length=1 << 16, n_groups=1, max_group_rows=8, max_shared=4000)
    need = abi.tss_prefix_attn_bytes(kv, 8, **sizes)
    if need:
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
            refused(prefix, abi.TSS_ENOSPACE, "tss_prefix_attn", kv, **sizes, **bad)
    assert abi.tss_prefix_attn_bytes(cache(head_dim=96), 8, **sizes) == 0
    assert abi.tss_prefix_attn_bytes(cache(), 7, **sizes) == 0


@pytest.mark.parametrize("kind", [abi.TSS_T_F16, abi.TSS_T_F32])
@pytest.mark.parametrize("rows,length", [(2, 32768), (2, 20000), (8, 32768), (3, 4096)])
def test_prefix_bounds_that_say_nothing(kind, rows, length):
    """The workspace holds a state of each row and head for every split.  Where max_shared covers the longest walk, as it
    does without bounds, the sequences' own pages are cut up as they are without a group."""
    kv = cache(n_kv_heads=32, head_dim=128, type=kind, n_seqs=rows, table_stride=2048, n_pages=1 << 16)

    def states(groups, shared):
        need = abi.tss_prefix_attn_bytes(kv, 32, rows, 1, length, groups, rows, shared)
        state = rows * 32 * (128 + 2) * 4
        assert need % state == 0
        return need // state or 1

    pages = length // 16
    alone, tight = states(0, 0), states(1, pages - 1)   # tight: one of the states is that of the one page left
    assert alone > 1 and tight > 1
    for shared in (pages, pages + 1, 2048):
        # a page more in the shared walk may take one split more or less
        assert states(1, shared) >= tight - 1 + alone - 1


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(n_groups=-1), dict(n_beams=0), dict(n_beams=33), dict(vocab=0), dict(row_stride=99),
    dict(n=0), dict(n=65, n_beams=32), dict(vocab=1, row_stride=1, n=4), dict(end_token=-1), dict(end_token=100),
    dict(logits=None), dict(scores=None), dict(score=None), dict(parent=None), dict(token=None), dict(logits=P + 2),
    dict(vocab=(1 << 20) + 1, row_stride=1 << 21), dict(n_groups=1 << 30)])
def test_beams_refuses(bad):
    refused(beams, abi.TSS_EINVAL, "tss_beam_select", **bad)


def test_beams_of_nothing_and_workspace():
    beams(n_groups=0, logits=None, scores=None)
    need = abi.tss_beam_select_bytes(2, 3, 100, 6)
    assert need > 0
    for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
        refused(beams, abi.TSS_ENOSPACE, "tss_beam_select", **bad)
    for bad in ((-1, 3, 100, 6), (2, 33, 100, 6), (2, 3, 0, 6), (2, 3, 100, 65), (2, 1, 5, 6)):
        assert abi.tss_beam_select_bytes(*bad) == 0


@pytest.mark.parametrize("bad", [dict(n_beams=0), dict(n_beams=33), dict(max_own=-1), dict(parents=None),
                                 dict(lengths=None)])
def test_reorder_refuses(bad):
    refused(reorder, abi.TSS_EINVAL, "tss_reorder_pages", **bad)


def test_reorder_tables():
    refused(reorder, abi.TSS_EINVAL, "tss_reorder_pages", cache(n_seqs=3))      # no multiple of the beams
    reorder(max_own=0)
    reorder(cache(n_seqs=0), parents=None, lengths=None)


@pytest.mark.parametrize("bad", [
    dict(pages=None), dict(type=abi.TSS_T_BF16), dict(type=7), dict(head_dim=96), dict(n_layers=0), dict(n_pages=0),
    dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(pages=P + 8), dict(page_table=None), dict(n_seqs=-2),
    dict(table_stride=0), dict(table_stride=1 << 28)])
def test_caches_refused(bad):
    for call in (append, prefix, reorder):
        refused(call, abi.TSS_EINVAL, "tss_", cache(**bad))


def test_numbers_that_do_not_fit():
    far = (1 << 32) + 5
    for call, names in ((append, ("layer", "n_q_heads", "type", "rows", "max_rows")),
                        (prefix, ("n_q_heads", "rows", "max_length", "n_groups", "max_group_rows", "max_shared")),
                        (beams, ("n_groups", "n_beams", "vocab", "end_token", "n")), (reorder, ("n_beams", "max_own"))):
        for name in names:
            for x in (far, 2.5):
                with pytest.raises(ValueError):
                    call(**{name: x})


@pytest.mark.parametrize("n", [0, -1, 65, (1 << 31) - 1])
def test_numbers_of_beams_refused_by_the_library(n):
    """Without a context the library refuses every call: no room is made first for more results than there can be."""
    with pytest.raises(abi.TSSError):
        abi.tss_get_beams(None, torch.zeros(100000, 2).numpy(), n)


def test_tensors_off_the_gpu_are_refused():
    pages, x = torch.zeros(1, 2, 2, 1, 16 * 64), torch.zeros(1, 1, 64)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        ops.append_kv(x, x, x, pages, i, i, i)
    with pytest.raises(ValueError):
        ops.prefix_attention(x, pages, i, i, i, i)
    with pytest.raises(ValueError):
        ops.beam_select(torch.zeros(2, 10), torch.zeros(1, 2), 4)
    with pytest.raises(ValueError):
        ops.reorder_pages(pages, i, i, i)


def test_frequencies():
    f = ops._frequencies(10000.0, 128)
    assert len(f) == 64 and f[0] == 1.0 and abs(f[32] - 0.01) < 1e-17 and f is ops._frequencies(10000.0, 128)


def test_rotations_refused():
    for rope in (0.0, -1.0, float("inf"), float("nan"), 5e-324, [1.0] * 63, [1.0] * 65, []):
        with pytest.raises(ValueError):
            ops._rotation(rope, 128)
    assert ops._rotation(None, 64) is None


def test_rotations_of_every_kind_of_number():
    want = list(ops._frequencies(500000.0, 64))
    for rope in (500000, 500000.0, torch.tensor(500000.0), torch.tensor(500000.0).numpy(), want,
                 torch.tensor(want, dtype=torch.float64)):
        assert list(ops._rotation(rope, 64)) == want
