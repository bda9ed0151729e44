"""Attention with a sliding window and sinks over the paged cache against a plain 64-bit form."""
import pytest
import torch

from paper_2609_26100_amd import ops
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16}


class Cache:
    """A pool whose unused slots and pages hold NaN, and each sequence's own K and V on the CPU."""

    def __init__(self, lengths, heads, hd, kind, seed, spare=3, layers=1, dead=None):
        g = torch.Generator().manual_seed(seed)
        t = TYPES[kind]
        self.kv = [tuple((a * torch.randn(n, heads, hd, generator=g)).to(t) for a in (1.0, 2.0)) for n in lengths]
        per = max(1, max(-(-n // 16) for n in lengths)) + 1
        total = len(lengths) * per + spare
        ids = torch.randperm(total, generator=g)[: len(lengths) * per].reshape(len(lengths), per)
        pool = torch.full((layers, total, 2, heads, 16 * hd), torch.nan, dtype=t)
        table = torch.full((len(lengths), per), -1, dtype=torch.int32)
        for s, (k, v) in enumerate(self.kv):
            n = k.shape[0]
            if not n:
                continue
            p = ops.pack_pages(k, v)
            if n % 16:
                kt, vt = p[-1, 0].view(heads, 16, hd), p[-1, 1].view(heads, 4, hd, 4)
                kt[:, n % 16:] = torch.nan
                for c in range(n % 16, 16):
                    vt[:, c // 4, :, c % 4] = torch.nan
            for i in range(p.shape[0]):
                pool[layers - 1, ids[s, i]] = p[i]
                table[s, i] = ids[s, i]
        if dead is not None:                 # pages given back: no row sees a token of theirs
            for s, i in dead:
                pool[layers - 1, table[s, i]] = torch.nan
                table[s, i] = [-1, total, 2 ** 31 - 1][i % 3]
        self.pool, self.table = pool.to(DEV), table.to(DEV)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device=DEV)


def queries(rows, heads, hd, kind, seed):
    g = torch.Generator().manual_seed(seed + 1000)
    return (1.5 * torch.randn(sum(rows), heads, hd, generator=g)).to(TYPES[kind])


def offsets(rows):
    return torch.tensor([0] + list(torch.tensor(rows).cumsum(0)), dtype=torch.int32, device=DEV)


def compare(got, q, rows, cache, sinks, window, scale=None):
    got = got.double().cpu()
    r0 = 0
    worst = 0.0
    for s, n in enumerate(rows):
        if n:
            k, v = cache.kv[s]
            see = ref.visible(n, k.shape[0], sinks, window)
            want, bound = ref.attention(q[r0:r0 + n], k, v, see, scale)
            err = (got[r0:r0 + n] - want).abs()
            assert torch.isfinite(got[r0:r0 + n]).all(), f"sequence {s}"
            over = (err / bound.clamp_min(1e-30)).where(err > 0, 0.0)
            worst = max(worst, float(over.max()))
            assert worst <= 1, f"sequence {s}: {worst} of the bound at {over.argmax()}"
        r0 += n
    return worst


CASES = [
    # lengths, rows, kv heads, group, hd, sinks, window
    ([1], [1], 1, 1, 64, 0, 0),
    ([1], [1], 2, 2, 128, 4, 1),
    ([16, 17, 15], [1, 1, 1], 2, 1, 128, 0, 16),
    ([40], [40], 2, 1, 64, 0, 0),
    ([33, 0, 5], [3, 0, 5], 2, 3, 128, 1, 1),
    ([200], [7], 4, 8, 128, 4, 33),
    ([1000, 3, 517], [1, 3, 9], 2, 4, 128, 4, 100),
    ([1000, 3, 517], [1, 3, 9], 2, 4, 64, 37, 64),
    ([2500], [1], 2, 1, 128, 4, 1024),
    ([2500, 2499, 2498, 2497], [2, 3, 4, 5], 2, 5, 128, 0, 0),
    ([700], [64], 2, 1, 128, 4, 100),
    ([700], [65], 2, 1, 64, 0, 7),
    ([700], [127], 3, 1, 128, 16, 0),
    ([300, 700], [300, 129], 2, 1, 128, 5, 50),
    ([650, 90], [600, 90], 1, 2, 128, 0, 256),
    ([400], [400], 2, 1, 64, 70, 1),
    ([513], [257], 2, 4, 128, 1, 300),
    ([90, 91], [16, 17], 40, 1, 128, 4, 32),
    ([5000], [33], 1, 1, 128, 100, 2000),
    ([130], [130], 2, 1, 128, 1000, 5),       # sinks beyond the length
    ([130], [30], 2, 1, 128, 0, 1 << 30),     # a window beyond the length
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("i", range(len(CASES)))
def test_window(kind, i):
    lengths, rows, heads, group, hd, sinks, window = CASES[i]
    c = Cache(lengths, heads, hd, kind, i)
    q = queries(rows, heads * group, hd, kind, i)
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, sinks, window)
    w = compare(out, q, rows, c, sinks, window)
    print(f"case {i} {kind}: {w:.3f} of the bound")
    # tight bounds of rows and length give the same up to the order of sums
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, sinks, window,
                               max_rows=max(rows), max_length=max(lengths))
    compare(out, q, rows, c, sinks, window)


@pytest.mark.parametrize("kind", list(TYPES))
def test_given_back_pages(kind):
    """Pages between the sinks and the window may be gone (ids outside the pool, memory of NaN)."""
    lengths, rows, sinks, window = [400, 333], [5, 20], 20, 64
    dead = [(s, i) for s, (n, r) in enumerate(zip(lengths, rows)) for i in range(2, (n - r - window + 1) // 16)]
    c = Cache(lengths, 2, 128, kind, 50, dead=dead)
    assert len(dead) > 20
    q = queries(rows, 4, 128, kind, 50)
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, sinks, window)
    compare(out, q, rows, c, sinks, window)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("sinks,window", [(0, 0), (5, 100), (40, 64), (200, 1), (0, 333)])
@pytest.mark.parametrize("group", [1, 3])
def test_many_blocks(hd, sinks, window, group):
    """More blocks of rows than run at once: longer blocks, ragged rows and lengths."""
    rows = [300, 65, 1, 0, 129, 200, 77, 32]
    c = Cache([411, 65, 700, 33, 129, 190, 500, 32], 16, hd, "f16", 58)
    q = queries(rows, 16 * group, hd, "f16", 58)
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, sinks, window)
    compare(out, q, rows, c, sinks, window)
    again = ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, sinks, window)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows_each", [3, 100])
def test_lost_page_hides_its_tokens(kind, rows_each):
    """A page id outside the pool inside the window: its tokens are as if they were not there."""
    n = 160
    c = Cache([n], 2, 64, kind, 51)
    c.table[0, 4] = -5
    q = queries([rows_each], 2, 64, kind, 51)
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets([rows_each]), c.lengths, 0, 0).double().cpu()
    see = ref.visible(rows_each, n, 0, 0)
    see[:, 64:80] = False
    want, bound = ref.attention(q, *c.kv[0], see)
    assert ((out - want).abs() <= bound).all()


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_that_see_nothing_and_rows_behind(kind):
    """More rows than tokens: the first see nothing and get zeros; rows behind the last sequence stay."""
    c = Cache([3, 40], 2, 128, kind, 52)
    rows = [7, 2]
    q = queries(rows + [4], 2, 128, kind, 52)
    out = torch.full((13, 2, 128), 7.0, dtype=TYPES[kind], device=DEV)
    ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, 1, 2, out=out)
    assert (out[9:] == 7).all() and (out[:4] == 0).all()
    see = ref.visible(3, 3, 1, 2)
    want, bound = ref.attention(q[4:7], *c.kv[0], see)
    assert ((out[4:7].double().cpu() - want).abs() <= bound).all()
    want, bound = ref.attention(q[7:9], *c.kv[1], ref.visible(2, 40, 1, 2))
    assert ((out[7:9].double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows", [[2, 2], [30, 30]])
def test_rows_that_see_nothing_where_others_are_split(kind, rows, monkeypatch):
    """A sequence without tokens beside a long one, whose pages are split: zeros, whatever the workspace held."""
    c = Cache([0, 3000], 2, 128, kind, 57)
    q = queries(rows, 2, 128, kind, 57)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).fill_(255 if k["dtype"] == torch.uint8 else 7))
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets(rows), c.lengths, 0, 0)
    assert (out[:rows[0]] == 0).all()
    want, bound = ref.attention(q[rows[0]:], *c.kv[1], ref.visible(rows[1], 3000, 0, 0))
    assert ((out[rows[0]:].double().cpu() - want).abs() <= bound).all()


def test_lengths_beyond_the_table_count_as_its_tokens():
    c = Cache([48], 2, 64, "f16", 53)
    c.table = c.table[:, :3].contiguous()
    q = queries([2], 2, 64, "f16", 53)
    want = ops.window_attention(q.to(DEV), c.pool, c.table, offsets([2]), c.lengths, 0, 20)
    got = ops.window_attention(q.to(DEV), c.pool, c.table, offsets([2]), c.lengths + 1000, 0, 20)
    assert torch.equal(got, want)
    capped = ops.window_attention(q.to(DEV), c.pool, c.table, offsets([2]), c.lengths, 0, 20, max_length=32)
    see = ref.visible(2, 32, 0, 20)
    ref_out, bound = ref.attention(q, c.kv[0][0][:32], c.kv[0][1][:32], see)
    assert ((capped.double().cpu() - ref_out).abs() <= bound).all()


def test_rows_beyond_max_rows_are_not_computed():
    c = Cache([50], 2, 64, "f16", 54)
    q = queries([9], 2, 64, "f16", 54)
    out = torch.full((9, 2, 64), 7.0, dtype=torch.float16, device=DEV)
    ops.window_attention(q.to(DEV), c.pool, c.table, offsets([9]), c.lengths, 0, 10, max_rows=4, out=out)
    want, bound = ref.attention(q, *c.kv[0], ref.visible(9, 50, 0, 10))
    assert ((out[:4].double().cpu() - want[:4]).abs() <= bound[:4]).all() and (out[4:] == 7).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows", [2, 70])
def test_strides_in_place_layer_and_scale(kind, rows):
    """Q and out inside wider rows, out = q, a layer other than the first, a scale of the caller's."""
    c = Cache([90], 2, 64, kind, 55, layers=3)
    q = queries([rows], 2, 64, kind, 55)
    wide = torch.full((rows, 200), 7.0, dtype=TYPES[kind], device=DEV)
    view = wide[:, 8:136].unflatten(1, (2, 64))
    view.copy_(q.to(DEV))
    ops.window_attention(view, c.pool, c.table, offsets([rows]), c.lengths, 2, 40, layer=2, scale=0.03, out=view)
    compare(view, q, [rows], c, 2, 40, scale=0.03)
    assert (wide[:, :8] == 7).all() and (wide[:, 136:] == 7).all()


@pytest.mark.parametrize("rows", [1, 130])
def test_large_pools(rows):
    """Pages beyond 4 GiB of a layer, and a layer beyond as much."""
    n, heads, hd = 2100, 8, 128
    pages = 80000                                                # 5.2 GB a layer
    pool = torch.full((2, pages, 2, heads, 16 * hd), torch.nan, dtype=torch.float16, device=DEV)
    g = torch.Generator().manual_seed(60)
    k, v = (torch.randn(n, heads, hd, generator=g).half() for _ in range(2))
    p = ops.pack_pages(k, v).to(DEV)
    ids = pages - 1 - torch.arange(p.shape[0]) * 7
    pool[1, ids.to(DEV)] = p
    q = queries([rows], heads, hd, "f16", 60)
    out = ops.window_attention(q.to(DEV), pool, ids.to(torch.int32)[None].to(DEV), offsets([rows]),
                               torch.tensor([n], dtype=torch.int32, device=DEV), 4, 1500, layer=1)
    want, bound = ref.attention(q, k, v, ref.visible(rows, n, 4, 1500))
    assert ((out.double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("kind", list(TYPES))
def test_masked_scores_that_overflow(kind):
    """K of tokens that a row does not see may be huge or not finite; what it sees may dominate completely."""
    c = Cache([100], 1, 64, kind, 61)
    k, v = c.kv[0]
    k[0:30] = 3e4 if kind == "f16" else 1e30
    k[30:40] = torch.inf
    k[60] = 30.0 * torch.sign(k[60])
    c.pool[0, c.table[0, :7].long()] = ops.pack_pages(k, v).to(DEV)
    q = queries([40], 1, 64, kind, 61)
    out = ops.window_attention(q.to(DEV), c.pool, c.table, offsets([40]), c.lengths, 0, 21)
    see = ref.visible(40, 100, 0, 21)
    want, bound = ref.attention(q, torch.where(k.abs() < 1e3, k, 0.0), v, see)
    assert ((out.double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("lengths,rows,window", [([3000], [1], 0), ([900, 40], [5, 2], 200), ([800], [300], 64)])
def test_captured_and_replayed(lengths, rows, window):
    """A captured call follows lengths, tables and queries that change between its replays."""
    c = Cache(lengths, 2, 128, "f16", 62)
    q = queries(rows, 4, 128, "f16", 62).to(DEV)
    off = offsets(rows)
    args = dict(sinks=4, window=window, max_rows=max(rows), max_length=max(lengths))
    ops.window_attention(q, c.pool, c.table, off, c.lengths, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.window_attention(q, c.pool, c.table, off, c.lengths, **args)
    for step in range(4):
        q.copy_(queries(rows, 4, 128, "f16", 70 + step))
        c.lengths.sub_(step)
        graph.replay()
        torch.cuda.synchronize()
        eager = ops.window_attention(q, c.pool, c.table, off, c.lengths, **args)
        assert torch.equal(out, eager) and torch.isfinite(out).all()


def test_the_same_bits_and_two_streams():
    cs = [Cache([4000], 2, 128, "f16", s) for s in (63, 64)]
    qs = [queries([2], 8, 128, "f16", s).to(DEV) for s in (63, 64)]

    def call(i):
        return ops.window_attention(qs[i], cs[i].pool, cs[i].table, offsets([2]), cs[i].lengths, 4, 3000)
    want = [call(0), call(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((i, call(i)))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i, o in got)


def test_refusals():
    c = Cache([40], 2, 64, "f16", 65)
    q = queries([2], 4, 64, "f16", 65).to(DEV)
    off = offsets([2])

    def call(q=q, pool=c.pool, table=c.table, off=off, lengths=c.lengths, **kw):
        return ops.window_attention(q, pool, table, off, lengths, **kw)
    for bad in (lambda: call(q=q.float()), lambda: call(q=q[:, :3]), lambda: call(q=q.transpose(0, 1)),
                lambda: call(pool=c.pool[:, ::2]), lambda: call(pool=c.pool.bfloat16()),
                lambda: call(table=c.table.long()), lambda: call(table=c.table[0]), lambda: call(off=off[:1]),
                lambda: call(lengths=c.lengths.cpu()), lambda: call(out=q[:1]), lambda: call(out=q.float())):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(sinks=-1), dict(window=-1), dict(layer=1), dict(scale=-1.0)):
        with pytest.raises(ops.abi.TSSError):
            call(**bad)
    with pytest.raises(ops.abi.TSSError):  # rows that are not aligned
        wide = torch.zeros(2, 300, dtype=torch.float16, device=DEV)
        call(q=wide[:, 4:260].unflatten(1, (4, 64)))


def test_scale_of_zero_is_refused():
    """None is 1 / sqrt(head_dim); a factor that is 0 in fp32 would be taken for it."""
    c = Cache([40], 2, 64, "f16", 66)
    q = queries([2], 4, 64, "f16", 66).to(DEV)
    for scale in (0.0, -0.0, 1e-50):
        with pytest.raises(ValueError):
            ops.window_attention(q, c.pool, c.table, offsets([2]), c.lengths, scale=scale)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows", [1, 40, 200])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", [300.0, 3e3, 3e4])
def test_scores_far_from_zero(kind, rows, sign, size):
    """Equal scores of any finite size: the mean of V, as at zero.  Scores of up to 6e10 times 1 / 8."""
    n, heads, hd = 250, 2, 64
    c = Cache([n], heads, hd, kind, 67)
    k, v = c.kv[0]
    k[:] = sign * size
    c.pool[0, c.table[0, :16].long()] = ops.pack_pages(k, v).to(DEV)
    q = torch.full((rows, heads, hd), size, dtype=TYPES[kind])
    got = ops.window_attention(q.to(DEV), c.pool, c.table, offsets([rows]), c.lengths, 0, 0).double().cpu()
    half = ref.HALF if kind == "f16" else ref.F32
    for r in range(rows):
        seen = v[: n - rows + r + 1].double()
        want = seen.mean(0)
        # equal weights (powers of two, exact), sums of n terms in fp32 and the roundings of 1 / L and of the result
        bound = n * ref.F32 * seen.abs().mean(0) * 2 + (half + 2 * ref.F32) * want.abs() + 2.0 ** -25
        assert ((got[r] - want).abs() <= bound).all(), (r, float((got[r] - want).abs().max()))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [1, 260])
def test_many_small_weights_beside_a_dominant_one(rows, hd):
    """A sink with nearly all of the weight and 20000 tokens of e^-18 of it each: together 3e-4, no less than they are.
    No splits: one workgroup walks all of a row's pages."""
    n, heads, seqs = 20000, 64, 4 if rows == 1 else 1
    g = torch.Generator().manual_seed(hd)
    k, v = torch.zeros(n, heads, hd), 4 + torch.randn(n, heads, hd, generator=g)
    k[0, :, 0] = 18.0
    v[0] = 0
    k, v = k.half(), v.half()
    pages = ops.pack_pages(k, v)[None].to(DEV)
    table = torch.arange(pages.shape[1], dtype=torch.int32, device=DEV).repeat(seqs, 1)
    q = torch.zeros(seqs * rows, heads, hd)
    q[:, :, 0] = hd ** 0.5
    lens = torch.full((seqs,), n, dtype=torch.int32, device=DEV)
    q = q.half()
    assert ops.abi.tss_window_attn_bytes(ops._cache(pages, table), heads, seqs * rows, rows, n, 0, 0) == 0
    got = ops.window_attention(q.to(DEV), pages, table, offsets([rows] * seqs), lens, max_rows=rows).double().cpu()
    for r, h in ((0, 0), (seqs * rows - 1, heads - 1), (rows // 2, 5)):
        see = torch.arange(n) <= (n - rows + r % rows)
        s = (q[r, h].double() @ k[:, h].double().T / hd ** 0.5).masked_fill(~see, -torch.inf)
        p = torch.softmax(s, 0)
        want = p @ v[:, h].double()
        # as ref.attention bounds it, but a weight's rounding in fp16 is at most 2^-32 of the largest: the scores are
        # exact (one product of two fp16 values and a power of two or 1/sqrt(128)), 18 log2 e and its exponent round
        pv, big = p @ v[:, h].double().abs(), float(v[:, h].abs().max())
        bound = 2 * (18 + 8) * 6 * ref.F32 * pv + 2 * n * ref.F32 * pv + ref.HALF * pv + n * 2.0 ** -32 * big \
            + ref.HALF * want.abs() + 2.0 ** -25
        err = (got[r, h] - want).abs()
        print(f"{rows} rows of {hd}: {float(err.max()):.3g}, bound {float(bound.min()):.3g}, output {float(want.min()):.3g}")
        assert (err <= bound).all()
