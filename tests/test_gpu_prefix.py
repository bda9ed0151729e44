"""Attention for sequences that share a prefix over the paged cache against a plain 64-bit form."""
import pytest
import torch

from paper_2609_26100_amd import ops
from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Groups:
    """Groups of sequences: (shared pages, [lengths]).  A pool whose unused slots and pages hold NaN; with `lone` only a
    group's first sequence knows the ids of the shared pages."""

    def __init__(self, groups, heads, hd, kind, seed, lone=True, layers=1, outside=()):
        g = torch.Generator().manual_seed(seed)
        t = TYPES[kind]
        self.shared = [s for s, _ in groups]
        self.kv, self.offsets = [], [0]
        of = []
        for s, lengths in groups:
            base = tuple((a * torch.randn(16 * s, heads, hd, generator=g)).to(t) for a in (1.0, 2.0))
            for n in lengths:
                more = max(0, n - 16 * s)
                own = tuple((a * torch.randn(more, heads, hd, generator=g)).to(t) for a in (1.0, 2.0))
                self.kv.append(tuple(torch.cat([b[:n], o]) for b, o in zip(base, own)))
                of.append((s, base))
            self.offsets.append(len(self.kv))
        for n in outside:
            self.kv.append(tuple(torch.randn(n, heads, hd, generator=g).to(t) for _ in range(2)))
            of.append((0, None))
        self.lengths = [k.shape[0] for k, _ in self.kv]
        width = max(max(self.shared + [0]), max(-(-n // 16) for n in self.lengths)) + 1
        total = sum(max(s, 1) for s in self.shared) + sum(-(-n // 16) for n in self.lengths) + 5
        ids = iter(torch.randperm(total, generator=g).tolist())
        pool = torch.full((layers, total, 2, heads, 16 * hd), torch.nan, dtype=t)
        self.table = torch.full((len(self.kv), width), -1, dtype=torch.int32)
        base_ids = {}
        for i, ((k, v), (s, base)) in enumerate(zip(self.kv, of)):
            first = i in self.offsets[:-1]
            if s and id(base) not in base_ids:
                mine = [next(ids) for _ in range(s)]
                base_ids[id(base)] = mine
                pool[layers - 1, mine] = ops.pack_pages(*base)
            if s and (first or not lone):
                self.table[i, :s] = torch.tensor(base_ids[id(base)], dtype=torch.int32)
            k, v = k[16 * s:], v[16 * s:]
            n = k.shape[0]
            if not n:
                continue
            p = ops.pack_pages(k, v)
            if n % 16:
                kt, vt = p[-1, 0].view(heads, 16, hd), p[-1, 1].view(heads, 4, hd, 4)
                kt[:, n % 16:] = torch.nan
                for c in range(n % 16, 16):
                    vt[:, c // 4, :, c % 4] = torch.nan
            for j in range(p.shape[0]):
                self.table[i, s + j] = next(ids)
                pool[layers - 1, self.table[i, s + j]] = p[j]
        self.pool, self.layer = pool, layers - 1


def queries(rows, heads, hd, kind, seed):
    g = torch.Generator().manual_seed(seed + 1000)
    return (1.5 * torch.randn(sum(rows), heads, hd, generator=g)).to(TYPES[kind])


def offsets(rows):
    return ints([0] + list(torch.tensor(rows).cumsum(0)))


def compare(got, q, rows, c, scale=None):
    got = got.double().cpu()
    r0 = 0
    for s, n in enumerate(rows):
        if n:
            k, v = c.kv[s]
            see = ref.visible(n, k.shape[0], 0, 0)
            want, bound = ref.attention(q[r0:r0 + n], k, v, see, scale)
            assert torch.isfinite(got[r0:r0 + n]).all(), f"sequence {s}"
            err = (got[r0:r0 + n] - want).abs()
            worst = float((err / bound.clamp_min(1e-30)).where(err > 0, 0.0).max())
            assert worst <= 1, f"sequence {s}: {worst} of the bound"
        r0 += n


def run(c, rows, q, **kw):
    return ops.prefix_attention(q.to(DEV), c.pool.to(DEV), c.table.to(DEV), offsets(rows), ints(c.lengths),
                                ints(c.shared), ints(c.offsets), layer=c.layer, **kw)


def check(groups, rows, heads, group, hd, kind, seed=0, scale=None, outside=(), lone=True, layers=1, **kw):
    c = Groups(groups, heads, hd, kind, seed, lone, layers, outside)
    q = queries(rows, heads * group, hd, kind, seed)
    got = run(c, rows, q, scale=scale, **kw)
    compare(got, q, rows, c, scale)
    return c, q, got


CASES = [
    # groups of (shared pages, lengths), rows, kv heads, group, hd
    ([(1, [17])], [1], 1, 1, 64),
    ([(1, [17, 18])], [1, 1], 2, 1, 128),
    ([(3, [49, 64, 65, 70])], [1, 1, 1, 1], 2, 2, 128),
    ([(2, [40, 33]), (0, [5, 1]), (7, [113, 160, 129])], [3, 1, 2, 1, 1, 20, 7], 2, 3, 64),
    ([(5, [81] * 16)], [1] * 16, 1, 1, 64),
    ([(5, [81 + i for i in range(17)])], [1] * 17, 1, 1, 128),
    ([(9, [150 + 7 * i for i in range(9)])], [2] * 9, 1, 8, 128),
    ([(20, [330, 321, 400]), (31, [500, 777])], [10, 1, 33, 4, 65], 2, 2, 128),
    ([(40, [645] * 30)], [5] * 30, 1, 1, 64),
    ([(63, [1009 + i for i in range(12)])], [1] * 12, 3, 4, 128),
    ([(200, [3300, 3201])], [1, 1], 1, 1, 64),
    ([(2, [33 + i for i in range(70)])], [1] * 70, 1, 2, 64),            # more sequences than a wave has lanes
]


@pytest.mark.parametrize("kind", ["f16", "f32"])
@pytest.mark.parametrize("case", CASES)
def test_against_64_bits(case, kind):
    check(*case, kind, seed=len(case[1]))


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_rows_inside_the_shared_pages(kind):
    """Pages that a row of the group does not see whole are read through each sequence's own table."""
    check([(4, [64, 80]), (6, [96, 100, 97])], [20, 3, 1, 30, 2], 2, 2, 64, kind, lone=False)
    check([(3, [10, 48, 60])], [10, 1, 2], 1, 2, 128, kind, lone=False)      # shorter than what is shared


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_empty_sequences_and_rows(kind):
    check([(2, [40, 33, 50])], [0, 2, 1], 2, 1, 64, kind)
    check([(0, [3, 0, 16])], [3, 0, 1], 1, 1, 128, kind)
    c = Groups([(2, [40, 33])], 1, 64, kind, 3, lone=False)      # more rows than tokens: the first see nothing
    rows = [45, 1]
    q = queries(rows, 2, 64, kind, 3)
    got = run(c, rows, q).cpu()
    assert not got[:5].any()
    compare(got[5:], q[5:], [40, 1], c)


def test_outside_every_group():
    check([(2, [40, 33]), (3, [60])], [1, 2, 3, 4, 1], 2, 2, 128, "f16", outside=(77, 20))
    c = Groups([(2, [40, 33])], 2, 64, "f16", 4, lone=False)
    q = queries([1, 2], 4, 64, "f16", 4)
    for offs, shared in (([0, 0], [2]), ([1, 2], [2]), ([5, 9], [2]), ([-3, 1], [2])):
        got = ops.prefix_attention(q.to(DEV), c.pool.to(DEV), c.table.to(DEV), offsets([1, 2]), ints(c.lengths),
                                   ints(shared), ints(offs))
        compare(got, q, [1, 2], c)
    got = ops.prefix_attention(q.to(DEV), c.pool.to(DEV), c.table.to(DEV), offsets([1, 2]), ints(c.lengths),
                               ints([]), ints([0]))
    compare(got, q, [1, 2], c)
    for shared in (-1, 0, 1, 2, 1000):                           # one group of all; beyond what is there
        if shared > 2:                                           # (2 pages are the same, the third is not)
            c.table[1, 2:] = c.table[0, 2:]
            c.kv[1] = tuple(torch.cat([a[:32], b[32:33]]) for a, b in zip(c.kv[1], c.kv[0]))
        got = ops.prefix_attention(q.to(DEV), c.pool.to(DEV), c.table.to(DEV), offsets([1, 2]), ints(c.lengths),
                                   ints([shared]))
        compare(got, q, [1, 2], c)


def test_many_groups():
    groups = [(1 + i % 3, [70 + i, 50]) for i in range(80)]
    check(groups, [1] * 160, 1, 2, 64, "f16")


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_bounds(kind):
    """Bounds that hold change nothing but the launch; tighter ones have their documented meaning."""
    groups, rows = [(6, [100, 110, 97]), (2, [40])], [3, 1, 2, 4]
    c = Groups(groups, 2, 128, kind, 5, lone=False)
    q = queries(rows, 4, 128, kind, 5)
    for kw in (dict(max_rows=4, max_length=112, max_shared=6, max_group_rows=6), dict(max_shared=3), dict(max_shared=0),
               dict(max_group_rows=3), dict(max_group_rows=0)):
        compare(run(c, rows, q, **kw), q, rows, c)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    run(c, rows, q, max_rows=2, out=out)
    assert (out[2:3] == 7).all() and (out[8:] == 7).all()
    compare(out[[3, 4, 5]], q[[3, 4, 5]], [0, 1, 2, 0], c)


@pytest.mark.parametrize("kind", ["f16", "f32"])
@pytest.mark.parametrize("rows", [[1, 2, 1], [3, 1, 40], [0, 1, 1]])
def test_long_own_pages_without_bounds(rows, kind):
    """Own pages in several splits beside those of the shared ones, where either kind is most of the walk."""
    check([(2, [5003, 3333]), (300, [4825])], rows, 2, 2, 64, kind, seed=17)
    check([(1, [2500, 20]), (0, [4000])], rows, 1, 4, 128, kind, seed=18)


def test_scale_strides_layers_and_rows_behind():
    c = Groups([(2, [40, 33])], 2, 64, "f16", 6, layers=3)
    buf = torch.zeros(6, 6 * 64 + 8, dtype=torch.float16, device=DEV)
    q = queries([1, 2], 4, 64, "f16", 6)
    view = buf.as_strided((6, 4, 64), (6 * 64 + 8, 64, 1))
    view[:3] = q.to(DEV)
    for scale in (None, 0.3, 1e-6):
        view[:3] = q.to(DEV)
        got = run(c, [1, 2], view, scale=scale, out=view)
        assert got.data_ptr() == view.data_ptr() and not view[3:].any()
        compare(got[:3], q, [1, 2], c, scale)


def test_beyond_four_gib():
    """Page ids whose bytes lie beyond 4 GiB, shared and own."""
    c = Groups([(3, [60, 49, 70])], 8, 128, "f16", 13, lone=False)
    q = queries([2, 1, 1], 16, 128, "f16", 13)
    want = run(c, [2, 1, 1], q)
    n = c.pool.shape[1]
    at = torch.randperm(n, generator=torch.Generator().manual_seed(1)) * (70000 // n)
    at[0] = 69999
    pool = torch.zeros(1, 70000, 2, 8, 16 * 128, dtype=torch.float16, device=DEV)          # 4.6 GB
    pool[0, at.to(DEV)] = c.pool[0].to(DEV)
    c.pool, c.table = pool, torch.where(c.table >= 0, at[c.table.long().clamp_min(0)].int(), -1)
    assert torch.equal(run(c, [2, 1, 1], q), want)


def test_special_values():
    """A dominant token in the prefix or behind it, scores far from zero, and infinities that no row sees."""
    c = Groups([(3, [60, 49])], 1, 64, "f16", 7)
    q = queries([2, 1], 1, 64, "f16", 7)
    for scale in (100.0, 3000.0, 1e7):
        compare(run(c, [2, 1], q, scale=scale), q, [2, 1], c, scale)


@pytest.mark.parametrize("kind", ["f16", "f32"])
@pytest.mark.parametrize("seqs", [1, 40, 128])          # blocks of 16, 64 and 128 rows
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", [30.0, 300.0, 3e3, 3e4])
def test_scores_far_from_zero(kind, seqs, sign, size):
    """Equal scores of any finite size, in shared and own pages: the mean of V, as at zero.  Up to 6e10 times 1 / 8."""
    shared, heads, hd = 14, 2, 64
    c = Groups([(shared, [16 * shared + 1 + i % 21 for i in range(seqs)])], heads, hd, kind, 14)
    for k, v in c.kv:
        k[:] = sign * size
    ids = c.table[c.table >= 0].unique().long()
    c.pool[0, ids, 0] = torch.where(c.pool[0, ids, 0].isnan(), torch.nan, sign * size).to(c.pool.dtype)
    q = torch.full((seqs, heads, hd), size, dtype=TYPES[kind])
    got = run(c, [1] * seqs, q).double().cpu()
    half = ref.HALF if kind == "f16" else ref.F32
    for i in range(seqs):
        v = c.kv[i][1].double()
        n, want = v.shape[0], v.mean(0)
        # equal weights (powers of two, exact), sums of n terms in fp32 and the roundings of 1 / L and of the result
        bound = n * ref.F32 * v.abs().mean(0) * 2 + (half + 2 * ref.F32) * want.abs() + 2.0 ** -25
        assert ((got[i] - want).abs() <= bound).all(), (i, float((got[i] - want).abs().max()))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("seqs", [2, 130, 256])         # blocks of 16, 64 and 128 rows, the last two of more than 64 pages
def test_many_small_weights_beside_a_dominant_one(seqs, hd):
    """A first shared token with nearly all of the weight, e^-18 of it for 20000 shared and a few own tokens each."""
    shared, heads = 1250, 16
    n = 16 * shared
    g = torch.Generator().manual_seed(hd + 1)
    k, v = torch.zeros(n + seqs * 3, heads, hd), 4 + torch.randn(n + seqs * 3, heads, hd, generator=g)
    k[0, :, 0] = 18.0
    v[0] = 0
    k, v = k.half(), v.half()
    own = [n + 3 * i for i in range(seqs)]                # three own tokens each, of which 1 + i % 3 are there
    lens = [n + 1 + i % 3 for i in range(seqs)]
    pages = torch.cat([ops.pack_pages(k[:n], v[:n])] + [ops.pack_pages(k[o:o + 3], v[o:o + 3]) for o in own])[None].to(DEV)
    table = torch.arange(shared + 1, dtype=torch.int32).repeat(seqs, 1)
    table[:, shared] = shared + torch.arange(seqs)
    q = torch.zeros(seqs, heads, hd)
    q[:, :, 0] = hd ** 0.5
    q = q.half()
    got = ops.prefix_attention(q.to(DEV), pages, table.to(DEV), offsets([1] * seqs), ints(lens), ints([shared]),
                               max_rows=1).double().cpu()
    for r, h in ((0, 0), (seqs - 1, heads - 1), (seqs // 2, 5)):
        m = lens[r] - n
        kr, vr = (torch.cat([x[:n, h], x[own[r]:own[r] + m, h]]).double() for x in (k, v))
        p = torch.softmax(q[r, h].double() @ kr.T / hd ** 0.5, 0)
        want, pv, big = p @ vr, p @ vr.abs(), float(vr.abs().max())
        # a weight's rounding in fp16 is at most 2^-32 of the largest: the scores are exact (one product of two fp16
        # values and a power of two or 1 / sqrt(128)), 18 log2 e and its exponent round; sums of n terms in fp32
        bound = 2 * (18 + 8) * 6 * ref.F32 * pv + 2 * n * ref.F32 * pv + ref.HALF * pv + n * 2.0 ** -32 * big \
            + ref.HALF * want.abs() + 2.0 ** -25
        assert ((got[r, h] - want).abs() <= bound).all(), (r, h, float(((got[r, h] - want).abs() / bound).max()))


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_equal_runs(kind):
    c = Groups([(30, [500, 520, 481]), (12, [200])], 2, 128, kind, 8)
    rows = [3, 1, 2, 9]
    q = queries(rows, 8, 128, kind, 8)
    a, b = run(c, rows, q), run(c, rows, q)
    assert torch.equal(a, b)


def test_captured_and_replayed():
    c = Groups([(9, [200, 220, 151]), (4, [80])], 2, 128, "f16", 9, lone=False)
    rows = [3, 1, 2, 9]
    q = queries(rows, 8, 128, "f16", 9)
    dq, pool, table, off, lens = q.to(DEV), c.pool.to(DEV), c.table.to(DEV), offsets(rows), ints(c.lengths)
    shared, offs = ints(c.shared), ints(c.offsets)
    ops.prefix_attention(dq, pool, table, off, lens, shared, offs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.prefix_attention(dq, pool, table, off, lens, shared, offs)
    for i, (cut, sh) in enumerate(((0, [9, 4]), (30, [8, 0]), (50, [3, 2]))):
        q = queries(rows, 8, 128, "f16", 10 + i)
        dq.copy_(q)
        lens.copy_(ints([n - cut for n in c.lengths]))
        shared.copy_(ints(sh))
        graph.replay()
        torch.cuda.synchronize()
        want = type("", (), {"kv": [tuple(x[: x.shape[0] - cut] for x in kv) for kv in c.kv]})
        compare(out, q, rows, want)


def test_two_graphs_and_a_stream():
    """Captured calls have workspaces of their own; a call on another stream is ordered by it alone."""
    c = Groups([(9, [200, 220, 151])], 2, 64, "f16", 11)
    qs = [queries([1, 1, 1], 8, 64, "f16", i) for i in (1, 2)]
    args = [c.pool.to(DEV), c.table.to(DEV), offsets([1, 1, 1]), ints(c.lengths), ints(c.shared)]
    dq = [q.to(DEV) for q in qs]
    outs, graphs = [], []
    for q in dq:
        ops.prefix_attention(q, *args)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(ops.prefix_attention(q, *args))
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for q, out in zip(qs, outs):
            compare(out, q, [1, 1, 1], c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = ops.prefix_attention(dq[0], *args)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, outs[0])


def test_refusals():
    c = Groups([(2, [40, 33])], 2, 64, "f16", 12)
    q = queries([1, 2], 4, 64, "f16", 12).to(DEV)
    ok = dict(q=q, pages=c.pool.to(DEV), page_table=c.table.to(DEV), row_offsets=offsets([1, 2]),
              lengths=ints(c.lengths), shared=ints([2]), group_offsets=ints([0, 2]))
    ops.prefix_attention(**ok)
    for bad in (dict(q=q.float()), dict(q=q[:, :3]), dict(shared=ints([2, 2])), dict(shared=2),
                dict(shared=ints([2, 2]), group_offsets=None), dict(shared=ints([2]).long()), dict(scale=0.0),
                dict(group_offsets=ints([0, 1, 2])), dict(out=q[:2]), dict(lengths=ints([40]))):
        with pytest.raises(ValueError):
            ops.prefix_attention(**dict(ok, **bad))
    for bad in (dict(layer=1), dict(scale=-1.0), dict(max_rows=-1), dict(max_shared=-1), dict(max_group_rows=-2)):
        with pytest.raises(ops.abi.TSSError):
            ops.prefix_attention(**dict(ok, **bad))
